"""Attention's sums over many keys of one weight, where every rounding of a running sum is to one side."""
import math

import pytest
import torch

from block_helpers import B, DEV, DTYPE, IO, U32, space

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("weight", [0.7, 0.3, 0.1])
def test_sums_over_many_keys(weight, dtype):
    """One key of score 0 and 65535 of log `weight`, by 520 images, so that none goes in parts."""
    N, Lq, Lk, D = 520, 100, 65536, 16
    size, flags = (N, Lq, Lk, 1, 1, D), IO[dtype]
    need = B.wino_cross_attention_workspace_bytes(*size, flags)
    assert need == 0
    t = DTYPE[dtype]
    q, k, v = (torch.zeros(s, dtype=t, device=DEV) for s in ((N, Lq, 1, D), (N, Lk, 1, D), (N, Lk, 1, D)))
    q[..., 0] = 1.0
    # two terms hold the score to 16 bits at least; what they hold is what counts
    high = torch.tensor(math.log(weight), dtype=torch.float64).to(t)
    low = torch.tensor(math.log(weight) - float(high), dtype=torch.float64).to(t)
    q[..., 1] = 1.0
    k[:, 1:, :, 0], k[:, 1:, :, 1] = high, low
    v[..., 0] = 1.0
    y, lse = torch.empty_like(q), torch.empty((N, 1, Lq), device=DEV)
    B.check(B.wino_cross_attention_nhwc(q, k, v, None, None, y, lse, *size, D, D, D, 1.0, flags))
    w = math.exp(float(high) + float(low))
    total = 1.0 + (Lk - 1) * w
    # a step's 32 keys of a lane, 1024 steps, the two halves; the exponent, exp2 and log2, and lse's own
    bound = (32 + Lk // 64 + 16) * U32 + abs(math.log(total)) * 4 * U32
    assert float((lse.double() - math.log(total)).abs().max()) <= bound
    if dtype != "f32":
        return
    # the backward pass of fp32 divides by a sum of its own
    dy, dq, dk, dv = torch.zeros_like(q), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    dy[..., 2] = 1.0
    need = B.wino_cross_attention_backward_workspace_bytes(*size, flags)
    assert need == 3 * ((N * Lq * 4 + 15) // 16 * 16)                # no parts here either
    B.check(B.wino_cross_attention_backward_nhwc(dy, q, k, v, y, lse, None, None, dq, dk, dv, *size, D, D, D, 1.0, flags,
                                                 space(need), need))
    want = torch.full((N, Lk), Lq * w / total, dtype=torch.float64, device=DEV)
    want[:, 0] = Lq / total
    # P's sum as above, P's exponent (below 20 in size) and exp2, products in six terms, sums of 100 rows
    bound = (32 + Lk // 64 + 16) * U32 + (20 * 4 + 8) * U32 + 2.0 ** -20 + (Lq + 16) * U32
    assert float(((dv[:, :, 0, 2].double() - want) / want).abs().max()) <= bound
    assert float(dq.abs().max()) <= 16 * U32 and float(dk.abs().max()) <= 16 * U32
