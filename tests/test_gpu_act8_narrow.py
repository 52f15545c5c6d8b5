"""8-bit checkpoints of channels whose range is a few units in the last place of their
centre.

With lo and hi an odd number m of units apart, centre rounds to one side by half a unit,
and one end lies (m + 1) / 2 units from it where half the range is m / 2: its quotient
passes 127, and the code is 127.  What is read back is then off by half a unit from the
centre's rounding, half a step from the code's and half a unit from the sum's; steps and
quotients add parts in 2^22 of half the range."""
import numpy as np
import pytest
import torch

import train_helpers as h
from oracle import train
from paper_1903_01521_amd import binding as B

pytestmark = pytest.mark.gpu

UNITS = [1, 2, 3, 5, 101, 201, 253, 255]
# in one launch, cut into chunks, one channel a lane
SHAPES = [(2, 5, 6, 16), (1, 150, 151, 8), (2, 9, 11, 9)]


def _narrow(shape, seed=0):
    """Channels of 1000 or -3 and up to UNITS[c] units in the last place, both ends taken."""
    N, H, W, C = shape
    rng = np.random.default_rng(seed)
    x = np.empty(shape, np.float32)
    for c in range(C):
        m = UNITS[c % len(UNITS)]
        base = np.float32(1000.0 if c % 3 else -3.0)
        steps = rng.integers(0, m + 1, (N, H, W))
        steps[:, 0, 0], steps[:, -1, -1] = 0, m
        x[..., c] = base + steps * np.abs(np.spacing(base))
    return x


def _check(q, x):
    N, H, W, C = x.shape
    codes, centre, step = h.split_ckpt(q, N, H, W, C)
    rcodes, rcentre, rstep = train.act8_pack(x)
    assert np.array_equal(centre, rcentre) and np.array_equal(step, rstep) and np.array_equal(codes, rcodes)


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_codes_stay_within_127(shape, offset):
    N, H, W, C = shape
    x = _narrow(shape)
    q = torch.full((B.wino_act8_bytes(N, C, H, W),), 85, dtype=torch.int8, device=h.DEV)
    wsb = B.wino_act8_workspace_bytes(N, C, H, W, 0)
    B.check(B.wino_act8_pack_nhwc(h.dev(x, offset=offset), q, N, C, H, W, 0, h.space(wsb), wsb))
    _check(q, x)
    v = h.like(h.dev(x))
    B.check(B.wino_act8_unpack_nhwc(q, v, N, C, H, W, 0))
    half = 0.5 * (x.max(axis=(1, 2)) - x.min(axis=(1, 2)))[:, None, None]
    bound = half / 254 + 1.0 * np.abs(np.spacing(x)) + half * 2.0 ** -22
    assert (np.abs(h.host(v) - x) <= bound).all()


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_the_norm_writes_them_too(shape):
    x = _narrow(shape, 1)
    C = shape[3]
    _, _, q = h.group_norm(x, np.ones(C), np.zeros(C), C, 1e-5, act="silu", ckpt=True)
    _check(q, x)
