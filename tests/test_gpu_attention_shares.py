"""fp16 attention keeps what is far below a row's largest score: its exponentials are held 2^7 times
as large, so that a share of 2^-20 has all its bits (2^-24 is fp16's least step, and 2^-14 the
least value with eleven)."""
import math

import numpy as np
import pytest

from block_helpers import B, IO, O, attend, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Lq,Lk,Hk", [(1, 127, 1), (40, 127, 1), (130, 127, 8), (1, 4096, 1), (40, 4096, 1)])
@pytest.mark.parametrize("share", [16.49, 16.51, 37.49, 128.49])
def test_small_shares_beside_the_largest(Lq, Lk, Hk, share):
    """Every 32nd key has score 0 and value 0, all others one score, whose exponential is `share` steps
    of 2^-24: rounded to whole steps all of them would be off to one side, by half a step."""
    D = 16
    score = math.log(share * 2.0 ** -24)
    first = float(np.float16(score))
    k, v = np.zeros((1, Lk, Hk, D)), np.zeros((1, Lk, Hk, D))
    small = np.arange(Lk) % 32 != 0
    k[0, small, :, 0], k[0, small, :, 1] = first, float(np.float16(score - first))
    v[0, small, :, 0], v[0, small, :, 1] = 1024.0, -513.0
    q = np.zeros((1, Lq, Hk, D))
    q[..., :2] = 1.0
    if Lk < 128:
        assert B.wino_cross_attention_workspace_bytes(1, Lq, Lk, Hk, Hk, D, IO["f16"]) == 0      # one part
    y, lse, _ = O.attention(q, k, v, 1.0, np.ones((1, Lk), bool))
    got, st = attend(q, k, v, 1.0, "f16")
    # scores are exact here (two terms), and the largest is 0; log2 e's rounding and the product's, of an
    # exponent below 21, exp2, and the sums over the keys; then P's own rounding and y's, 2^-11 each, and
    # what falls below 2^-32 of the largest
    rel = (21 * 2 + 4 + Lk + 8) * 2.0 ** -24
    tol = np.abs(y) * (2 * rel + 2.0 ** -11 + 2.0 ** -32 / math.exp(score) + 2.0 ** -11)
    within(got, y, tol + 2.0 ** -25, "y")
    within(st, lse, np.full(lse.shape, 2 * rel) + np.abs(lse) * 2.0 ** -22, "lse")
    # the share in whole steps would be past the bound
    assert abs(share - round(share)) / share * np.abs(y).max() > 2 * (tol.max() + 2.0 ** -25)
