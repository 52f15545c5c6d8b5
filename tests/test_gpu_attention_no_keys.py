"""Images without keys whose queries or gradients are not finite: y = 0, lse = -infinity and
zero gradients, whether a length or a mask left nothing."""
import numpy as np
import pytest

from block_helpers import attend, attend_back, host
from train_helpers import rounded

pytestmark = pytest.mark.gpu

# few rows and many; keys in parts and whole; vectors of whole words and of none
SIZES = [(3, 40, 150, 2, 2, 64, 0), (3, 3, 150, 2, 1, 64, 0), (3, 2, 900, 2, 1, 128, 0), (3, 40, 900, 1, 1, 40, 1),
         (3, 130, 70, 2, 2, 20, 0)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("junk", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("size", SIZES)
def test_images_without_keys(size, junk, dtype):
    N, Lq, Lk, Hq, Hk, D, offset = size
    rng = np.random.default_rng(91)
    q, dy = (rounded(rng.standard_normal((N, Lq, Hq, D)), dtype) for _ in "ab")
    k, v = (rounded(rng.standard_normal((N, Lk, Hk, D)), dtype) for _ in "ab")
    klen, mask = [Lk - 5, Lk, 0], rng.integers(0, 2, (N, Lk))
    mask[0, 0], mask[1] = 1, 0
    clean, _ = attend(q, k, v, 0.25, dtype, klen, mask, offset=offset)
    lse = host(_)
    grads = attend_back(dy, q, k, v, host(clean), lse, 0.25, dtype, klen, mask, offset=offset)
    q2, dy2 = q.copy(), dy.copy()
    q2[1:, 1, :, 3], dy2[1:, Lq - 1, 0, 5] = junk, junk
    y, st = attend(q2, k, v, 0.25, dtype, klen, mask, offset=offset)
    assert (host(y)[1:] == 0).all() and np.isneginf(host(st)[1:]).all()
    assert np.array_equal(host(y)[0], host(clean)[0]) and np.array_equal(host(st)[0], lse[0])
    for g, c in zip(attend_back(dy2, q2, k, v, host(y), host(st), 0.25, dtype, klen, mask, offset=offset), grads):
        assert (host(g[0])[1:] == 0).all() and np.array_equal(host(g[0])[0], host(c[0])[0])
