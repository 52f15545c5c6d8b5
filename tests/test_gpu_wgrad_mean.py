"""The weight gradient of a layer whose input is formed from the norm of x, with means
thousands of spreads away: as close as at a mean of zero, for the statistics given.

Bound, u = 2^-24: n is off by 2u |n| (x - mean, the product with rstd), z by that times
gamma, 3u |n gamma| and u |z|, SiLU by 1.1 of it and (2 |z| + 8) u of itself; an operand's
two fp16 terms by 2^-22 of it and 2^-38 of 2 |gamma| sqrt(D H W) + |beta|; a product by
2^-22 more from each operand and the term left out; the sums by SUM."""
import numpy as np
import pytest
import torch

import train_helpers as h
from oracle import train
from paper_1903_01521_amd import binding as B

pytestmark = pytest.mark.gpu

EPS, U = 1e-5, h.U32


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("mean", [0.0, 3000.0])
@pytest.mark.parametrize("shape,G", [((2, 14, 13, 40, 24), 8), ((8, 9, 10, 64, 130), 16), ((1, 30, 31, 70, 64), 1)])
def test_means_far_from_zero(shape, G, mean, act):
    N, H, W, C, K = shape
    rng = np.random.default_rng(1)
    x = (mean + rng.standard_normal((N, H, W, C)) * np.exp(0.3 * rng.standard_normal(C))).astype(np.float32)
    dy = np.abs(rng.standard_normal((N, H, W, K))).astype(np.float32)     # so that one sign of an error adds up
    gamma = (1 + 0.2 * rng.standard_normal(C)).astype(np.float32).astype(np.float64)
    beta = (0.5 * rng.standard_normal(C)).astype(np.float32).astype(np.float64)
    st = np.stack(train.group_stats(x, G, EPS), -1).astype(np.float32).astype(np.float64)
    n = train.normed(x, st[..., 0], st[..., 1])
    z = n * gamma + beta
    a = train.act(z, act)
    off = 1.1 * (5 * U * np.abs(n * gamma) + U * np.abs(z)) + (np.abs(a) * (2 * np.abs(z) + 8) * U if act == "silu" else 0)
    off += 2.0 ** -38 * (2 * np.abs(gamma).max() * np.sqrt(C // G * H * W) + np.abs(beta).max())
    flags = h.ACT[act]
    dg = torch.full((K, C, 3, 3), float("nan"), device=h.DEV)
    wsb = B.wino_conv2d_wgrad_workspace_bytes(N, C, H, W, K, 1, flags)
    B.check(B.wino_conv2d_wgrad_nhwc(h.dev(x), h.dev(dy), dg, h.dev(st), h.dev(gamma), h.dev(beta), G, N, C, H, W, K, 1,
                                     flags, h.space(wsb), wsb))
    bound = train.wgrad(off, dy, 1) + (3 * 2.0 ** -22 + h.SUM) * train.wgrad(np.abs(a), dy, 1)
    bound += 2.0 ** -38 * dy.max() * train.wgrad(np.abs(a), np.ones_like(dy), 1)
    miss = np.abs(h.host(dg) - train.wgrad(a, dy, 1))
    assert (miss <= bound).all(), float((miss / bound).max())
