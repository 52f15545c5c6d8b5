"""The fp64 references of the training calls against differences and an
independent form (CPU only)."""
import numpy as np
import pytest

from oracle import direct, train

EPS = 1e-5


def _inputs(seed, N=2, H=3, W=4, C=6):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((N, H, W, C)), 1.0 + 0.3 * rng.standard_normal(C), 0.3 * rng.standard_normal(C),
            rng.standard_normal((N, H, W, C)))


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
@pytest.mark.parametrize("G", [1, 2, 6])
def test_group_norm_gradients_match_differences(kind, G):
    x, gamma, beta, dy = _inputs(3 + G)
    _, mean, rstd = train.group_norm(x, gamma, beta, G, EPS, kind)
    dx, dgamma, dbeta = train.group_norm_backward(dy, x, mean, rstd, gamma, beta, kind)

    def loss(x, gamma, beta):
        return float((train.group_norm(x, gamma, beta, G, EPS, kind)[0] * dy).sum())
    # central differences: the error is h^2 (third derivatives, here below 1e3) and rounding / h
    h = 1e-5
    rng = np.random.default_rng(0)
    for value, grad, slot in ((x, dx, 0), (gamma, dgamma, 1), (beta, dbeta, 2)):
        for _ in range(8):
            i = tuple(int(rng.integers(n)) for n in value.shape)
            args = [[x, gamma, beta], [x, gamma, beta]]
            for a, step in zip(args, (h, -h)):
                moved = value.copy()
                moved[i] += step
                a[slot] = moved
            assert abs((loss(*args[0]) - loss(*args[1])) / (2 * h) - grad[i]) < 1e-6


def test_weight_gradient_matches_differences():
    # the layer is linear in its filters: dg is the difference of sum(conv(a, g) dy)
    rng = np.random.default_rng(1)
    a = rng.standard_normal((2, 5, 6, 3)).astype(np.float32)
    for pad in (0, 1, 2):
        dy = rng.standard_normal((2, 3 + 2 * pad, 4 + 2 * pad, 4))
        dg = train.wgrad(a, dy, pad)
        for k, c, r, s in ((0, 0, 0, 0), (3, 2, 2, 2), (1, 1, 0, 2), (2, 0, 1, 1)):
            g = np.zeros((4, 3, 3, 3), np.float32)
            g[k, c, r, s] = 1.0
            y = direct.conv2d(np.ascontiguousarray(a.transpose(0, 3, 1, 2)), g, pad).transpose(0, 2, 3, 1)
            assert abs((y * dy).sum() - dg[k, c, r, s]) < 1e-9


def test_checkpoint_error_is_half_a_step():
    rng = np.random.default_rng(2)
    x = (rng.standard_normal((3, 7, 5, 9)) * np.exp(rng.standard_normal(9))).astype(np.float32)
    x[0, :, :, 3] = 2.5                                  # a constant channel
    codes, centre, step = train.act8_pack(x)
    v = train.act8_unpack(codes, centre, step)
    bound = 0.5 * step[:, None, None] + 2.0 ** -22 * np.abs(x).max()
    assert (np.abs(v - x) <= bound).all()
    assert step[0, 3] == 0 and (v[0, :, :, 3] == 2.5).all()
    assert codes.min() == -127 and codes.max() == 127
