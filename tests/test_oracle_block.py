"""The 64-bit formulas of the attention half: gradients against differences, shared heads
against repeated ones, rotations that keep lengths and depend on distances alone."""
import numpy as np
import pytest

from oracle import block as O

RNG = np.random.default_rng


def slope(f, x, g, h=1e-5):
    """The derivative of sum f(x) g along a random direction, by central differences."""
    d = RNG(7).standard_normal(x.shape)
    return ((f(x + h * d) - f(x - h * d)) * g).sum() / (2 * h), d


# h^2 of a third derivative of order 1..100 and 1e-16 / h of values of order 1..100
CLOSE = 1e-7


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("D,R", [(8, 8), (7, 4), (5, 0)])
def test_norm_gradients(D, R, pairs):
    rng = RNG(1)
    x, dy, gamma = rng.standard_normal((2, 3, 2, D)), rng.standard_normal((2, 3, 2, D)), 1 + 0.2 * rng.standard_normal(D)
    angle = rng.uniform(0, 6, (2, 3, 1, R // 2))
    c, s = np.cos(angle), np.sin(angle)
    dx, dg, _ = O.head_norm_backward(dy, x, gamma, c, s, 1e-3, pairs)
    want, d = slope(lambda v: O.head_norm(v, gamma, c, s, 1e-3, pairs), x, dy)
    assert abs((dx * d).sum() - want) < CLOSE * max(1, abs(want))
    want, d = slope(lambda v: O.head_norm(x, v, c, s, 1e-3, pairs), gamma, dy)
    assert abs((dg * d).sum() - want) < CLOSE * max(1, abs(want))


@pytest.mark.parametrize("pairs", [False, True])
def test_rotation_is_of_distances(pairs):
    rng = RNG(2)
    q, k, freq = rng.standard_normal(8), rng.standard_normal(8), rng.uniform(0.1, 1, 4)

    def at(x, t):
        return O.turn(x, np.cos(freq * t), np.sin(freq * t), pairs)
    assert np.allclose(np.linalg.norm(at(q, 5)), np.linalg.norm(q), rtol=1e-14)
    assert np.allclose(at(q, 9) @ at(k, 4), at(q, 105) @ at(k, 100), rtol=1e-12)


@pytest.mark.parametrize("Hq,Hk", [(2, 2), (4, 2), (3, 1)])
def test_attention_gradients(Hq, Hk):
    rng = RNG(3)
    N, Lq, Lk, D = 3, 4, 6, 5
    q, k, v = (rng.standard_normal((N, n, h, D)) for n, h in ((Lq, Hq), (Lk, Hk), (Lk, Hk)))
    dy = rng.standard_normal((N, Lq, Hq, D))
    kept = O.kept_keys(N, Lk, [6, 0, 4], rng.integers(0, 2, (N, Lk)) | (np.arange(Lk) == 0))
    y, lse, p = O.attention(q, k, v, 0.4, kept)
    assert np.all(y[1] == 0) and np.all(np.isneginf(lse[1])) and np.allclose(p[0].sum(-1), 1)
    got = O.attention_backward(dy, q, k, v, y, lse, 0.4, kept)[:3]
    for i, x in enumerate((q, k, v)):
        def f(u):
            a = [q, k, v]
            a[i] = u
            return O.attention(*a, 0.4, kept)[0]
        want, d = slope(f, x, dy)
        assert abs((got[i] * d).sum() - want) < CLOSE * max(1, abs(want))
    assert np.all(got[0][1] == 0) and np.all(got[1][1] == 0) and np.all(got[2][~kept] == 0)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_gated_gradients(act):
    rng = RNG(4)
    x, w, b, dy = (rng.standard_normal(s) for s in ((5, 4), (2, 3, 4), (2, 3), (5, 3)))
    got = O.gated_backward(dy, x, w, b, act)[:3]
    for i, v in enumerate((x, w, b)):
        def f(u):
            a = [x, w, b]
            a[i] = u
            return O.gated(*a, act)[0]
        want, d = slope(f, v, dy)
        assert abs((got[i] * d).sum() - want) < CLOSE * max(1, abs(want))
