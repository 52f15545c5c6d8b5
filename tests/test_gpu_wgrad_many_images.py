"""The weight gradient from checkpoints of many small images, whose rows take a workgroup
several turns to bound: magnitudes that differ by image and by channel, on the bounds of
test_gpu_wgrad_scale.py."""
import numpy as np
import pytest

import test_gpu_wgrad_scale as scale
import train_helpers as h
from oracle import train

pytestmark = pytest.mark.gpu

U = h.U32


@pytest.mark.parametrize("shape", [(300, 2, 3, 9, 20, 1), (4100, 1, 2, 5, 3, 1), (66, 3, 3, 1100, 17, 1)], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_from_the_checkpoint(shape, dtype):
    N, H, W, C, K, pad = shape
    x, dy, _, _, rng = scale._inputs(shape, dtype, -30, -30, 6)
    x = h.rounded(x * 2.0 ** rng.integers(-12, 1, (N, 1, 1, 1)), dtype)
    x[N // 2] = h.rounded(x[N // 2] * 2.0 ** 20, dtype)             # the largest are one image's
    codes, centre, step = train.act8_pack(x)
    a = train.act8_unpack(codes, centre, step)
    most = (np.abs(centre) + 127.0 * step).max(axis=0).astype(np.float64)
    off_a = 4 * U * (np.abs(codes * step[:, None, None].astype(np.float64)) + np.abs(centre)[:, None, None])
    dg = scale._call(h.make_ckpt(codes, centre, step), dy, pad, dtype, (N, C, H, W, K), ckpt=True)
    scale._check(dg, a, dy, pad, most, scale._most(dy), off_a)
