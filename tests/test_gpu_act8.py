"""The 8-bit activation checkpoint against the oracle: codes and rows are equal,
read-back values within fp32 rounding."""
import numpy as np
import pytest
import torch

import train_helpers as h
from oracle import train
from paper_1903_01521_amd import binding as B

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1, 1, 1), (2, 1, 1, 20), (2, 5, 3, 7), (3, 13, 7, 40), (2, 28, 28, 128), (1, 150, 151, 8), (1, 131, 77, 33),
          (1, 3, 5, 2100), (2, 130, 129, 24)]


def _x(shape, dtype, seed=0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape) * np.exp(rng.standard_normal(shape[3])) + rng.standard_normal(shape[3])
    return h.rounded(x, dtype)


def _pack(x, dtype, offset=0):
    N, H, W, C = x.shape
    q = torch.full((B.wino_act8_bytes(N, C, H, W),), 85, dtype=torch.int8, device=h.DEV)
    wsb = B.wino_act8_workspace_bytes(N, C, H, W, h.IO[dtype])
    B.check(B.wino_act8_pack_nhwc(h.dev(x, dtype, offset), q, N, C, H, W, h.IO[dtype], h.space(wsb), wsb))
    return q


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_pack_and_unpack(shape, dtype, offset):
    N, H, W, C = shape
    x = _x(shape, dtype)
    q = _pack(x, dtype, offset)
    codes, centre, step = h.split_ckpt(q, N, H, W, C)
    rcodes, rcentre, rstep = train.act8_pack(x)
    assert np.array_equal(centre, rcentre) and np.array_equal(step, rstep) and np.array_equal(codes, rcodes)
    v = h.dev(np.full(shape, np.nan), dtype, offset)
    B.check(B.wino_act8_unpack_nhwc(q, v, N, C, H, W, h.IO[dtype]))
    ref = train.act8_unpack(rcodes, rcentre, rstep)
    bound = 4 * h.U32 * (np.abs(ref) + np.abs(rcentre)[:, None, None]) + h.HALF_ULP[dtype] * np.abs(ref)
    assert (np.abs(h.host(v) - ref) <= bound).all()


@pytest.mark.parametrize("shape,G", [((2, 13, 7, 40), 8), ((1, 150, 151, 8), 2), ((1, 131, 77, 33), 3)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_norm_writes_the_same_checkpoint(shape, G, dtype):
    N, H, W, C = shape
    x = _x(shape, dtype, 1)
    q = _pack(x, dtype)
    _, _, fused = h.group_norm(x, np.ones(C), np.zeros(C), G, 1e-5, dtype, "silu", ckpt=True)
    n = N * H * W * C
    assert torch.equal(q[:n], fused[:n]) and torch.equal(q[(n + 15) // 16 * 16:], fused[(n + 15) // 16 * 16:])


def test_extreme_ranges():
    x = np.zeros((1, 2, 2, 8), np.float32)
    x[..., 0] = 5.0                                     # constant
    x[..., 1].flat[:] = [3e38, -3e38, 0.0, 1e38]        # the range passes fp32's largest value
    x[..., 2].flat[:] = [1e-38, 0.0, -1e-38, 0.0]       # below 2^-100: its centre, 0
    x[..., 3].flat[:] = [np.inf, 0.0, 1.0, 2.0]
    x[..., 4].flat[:] = [np.nan, 0.0, 1.0, 2.0]
    x[..., 5].flat[:] = [-np.inf, np.inf, 1.0, 2.0]
    x[..., 6].flat[:] = [1.0, 2.0, 3.0, 4.0]
    q = _pack(x, "f32")
    v = torch.zeros(x.shape, device=h.DEV)
    B.check(B.wino_act8_unpack_nhwc(q, v, 1, 8, 2, 2, 0))
    v = h.host(v)[0].reshape(4, 8)
    assert (v[:, 0] == 5.0).all() and (v[:, 2] == 0.0).all() and (v[:, 7] == 0.0).all()
    assert np.abs(v[:, 1] / 3e38 - x[0].reshape(4, 8)[:, 1] / 3e38).max() < 1.01 / 254
    assert np.isnan(v[:, 3:6]).all()
    assert np.abs(v[:, 6] - [1, 2, 3, 4]).max() <= 3 / 508 + 1e-6
