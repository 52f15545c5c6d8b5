"""Channels of the norm that are not turned stand alone: what is not finite in one of them
reaches no other through the rotation."""
import numpy as np
import pytest

from block_helpers import host
from test_gpu_qk_norm import call, make

pytestmark = pytest.mark.gpu

# N, Lq, Lk, Hq, Hk, D, R: from one to eight pairs a lane
SIZES = [(1, 5, 6, 2, 1, 64, 32), (2, 3, 4, 3, 2, 40, 8), (1, 6, 3, 2, 2, 7, 4), (1, 4, 4, 5, 1, 12, 4), (1, 7, 2, 1, 1, 10, 0)]


def others(a, b, channel):
    """Every channel but one is the same in a and b."""
    kept = np.arange(a.shape[-1]) != channel
    return np.array_equal(a[..., kept], b[..., kept])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("size", SIZES)
def test_channels_that_are_not_turned(size, pairs, dtype):
    R, D = size[6], size[5]
    for at in sorted({R, R + 1, D - 1}):
        d = make(size, dtype, 92, 0)
        clean, grads = ([host(t) for t in call(d, size, dtype, pairs, back=back)] for back in (False, True))

        # gamma: y of its own channel alone, and nothing of dgamma
        gamma = d["gq"].copy()
        d["gq"][at] = np.inf
        y = host(call(d, size, dtype, pairs)[0])
        assert others(y, clean[0], at) and np.isinf(y[..., at]).all()
        dgamma = host(call(d, size, dtype, pairs, back=True)[2])
        assert np.array_equal(dgamma, grads[2])
        d["gq"] = gamma

        # x: its head over an infinite root mean square is zero, and NaN where it was
        x = d["q"].copy()
        d["q"][0, 1, 0, at] = -np.inf
        y = host(call(d, size, dtype, pairs)[0])
        head = y[0, 1, 0].copy()
        assert np.isnan(head[at]) and (head[np.arange(D) != at] == 0).all()
        y[0, 1, 0] = clean[0][0, 1, 0]
        assert np.array_equal(y, clean[0])
        d["q"] = x

        # dy: dgamma of its own channel alone, and dx of its head
        d["dyq"][0, 1, 0, at] = np.inf
        got = [host(t) for t in call(d, size, dtype, pairs, back=True)]
        assert others(got[2], grads[2], at) and np.isinf(got[2][at])
        got[0][0, 1, 0] = grads[0][0, 1, 0]
        assert np.array_equal(got[0], grads[0])
