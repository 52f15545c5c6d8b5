"""Sums of the norm and its gradients over 2^30 values: within SUM of the sums of absolute
values, 256 roundings, whatever the size.

The values are one number but for 256 zeros an image, the case in which every rounding of
a long 32-bit sum may go the same way (4096 terms in turn: 6e-5).  The zeros come first,
so that each thread's first value is the one that is far from all others: squares about it
are 64 times what they are about the mean in a part of 64 values, whose sum is 64 roundings
off and has as much subtracted, 2^-11 of the variance and half of that of rstd."""
import pytest
import torch

import train_helpers as h
from paper_1903_01521_amd import binding as B

pytestmark = pytest.mark.gpu


def test_sums_do_not_lose_more_with_the_size():
    N, H, W = 1024, 1024, 1024
    v = 1.0159916877746582
    assert float(torch.tensor(v)) == v
    x = torch.full((N, H, W, 1), v, device=h.DEV)
    x.view(N, H * W)[:, :256] = 0.0
    filled = H * W - 256
    # forward: the mean against its own value
    y, st = torch.empty_like(x), torch.zeros((N, 1, 2), device=h.DEV)
    wsb = B.wino_group_norm_workspace_bytes(N, 1, H, W, 1, 0)
    B.check(B.wino_group_norm_nhwc(x, None, None, y, st, None, N, 1, H, W, 1, 0.0, 0, h.space(wsb), wsb))
    share = filled / (H * W)
    assert float((st[..., 0].double() - v * share).abs().max()) <= h.SUM * v
    var = v * v * share * (1 - share)
    assert float((st[..., 1].double() * var ** 0.5 - 1).abs().max()) <= 2.0 ** -12 + h.SUM
    # backward with n = x: dbeta the sum of dy, dgamma that of dy x
    st[..., 0], st[..., 1] = 0.0, 1.0
    dgamma, dbeta = torch.zeros(1, device=h.DEV), torch.zeros(1, device=h.DEV)
    wsb = B.wino_group_norm_backward_workspace_bytes(N, 1, H, W, 1, 0)
    B.check(B.wino_group_norm_backward_nhwc(x, x, st, None, None, y, dgamma, dbeta, N, 1, H, W, 1, 0, h.space(wsb), wsb))
    assert abs(float(dbeta) / (N * filled * v) - 1) <= h.SUM
    assert abs(float(dgamma) / (N * filled * v * v) - 1) <= h.SUM
    # dx = dy - m1 - x m2, m1 and m2 within SUM
    m1, m2 = v * share, v * v * share
    for at, dy in ((0, 0.0), (-1, v)):
        dx = y.view(N, H * W)[:, at].double()
        assert float((dx - (dy - m1 - dy * m2)).abs().max()) <= h.SUM * (m1 + v * m2) + 8 * h.U32 * (1 + v) ** 3


def test_sums_of_many_chunks_and_images():
    # 2^12 chunks of an image, and 2^13 images of a few pixels: the joins of the parts
    for N, H, W in ((1, 4096, 4096), (8192, 8, 8)):
        v = 1.0159916877746582
        dy = torch.full((N, H, W, 4), v, device=h.DEV)
        x = torch.ones_like(dy)
        st = torch.zeros((N, 1, 2), device=h.DEV)
        st[..., 1] = 1.0
        dx = torch.empty_like(dy)
        dgamma, dbeta = torch.zeros(4, device=h.DEV), torch.zeros(4, device=h.DEV)
        wsb = B.wino_group_norm_backward_workspace_bytes(N, 4, H, W, 1, 0)
        B.check(B.wino_group_norm_backward_nhwc(dy, x, st, None, None, dx, dgamma, dbeta, N, 4, H, W, 1, 0, h.space(wsb),
                                                wsb))
        for d in (dgamma, dbeta):
            assert float((d.double() / (N * H * W * v) - 1).abs().max()) <= h.SUM
