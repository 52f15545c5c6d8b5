"""The training calls' sizes and refusals: arguments are checked before any HIP call
(CPU only: no call here reaches a kernel)."""
import pytest

from paper_1903_01521_amd import binding as B

FAKE = 0x100000000                     # never dereferenced: every call here is refused
MAX = 2**64 - 1
INV, UNS, WS = B.WINO_ERR_INVALID_ARG, B.WINO_ERR_UNSUPPORTED, B.WINO_ERR_WORKSPACE


def at(i):
    return FAKE + (i << 40)


def test_checkpoint_bytes():
    assert B.wino_act8_bytes(2, 5, 3, 7) == (2 * 5 * 3 * 7 + 15) // 16 * 16 + 2 * 5 * 8
    assert B.wino_act8_bytes(64, 256, 56, 56) == 64 * 256 * 56 * 56 + 64 * 256 * 8
    for bad in ((0, 5, 3, 7), (2, 0, 3, 7), (2, 5, -1, 7), (2, 5, 3, 0), (2**31 - 1, 2**31 - 1, 2, 2)):
        assert B.wino_act8_bytes(*bad) == 0


def test_workspace_bytes():
    # a group of the image fits the registers: none; else parts and statistics
    assert B.wino_group_norm_workspace_bytes(8, 128, 28, 28, 32, 0) == 0
    assert B.wino_group_norm_workspace_bytes(1, 64, 512, 512, 1, 0) > 0
    assert B.wino_group_norm_backward_workspace_bytes(8, 128, 28, 28, 32, 0) >= 8 * 128 * 8
    assert B.wino_conv2d_wgrad_workspace_bytes(1, 32, 56, 56, 32, 1, 0) >= 9 * 32 * 32 * 4
    for f in (B.wino_group_norm_workspace_bytes, B.wino_group_norm_backward_workspace_bytes):
        assert f(8, 128, 28, 28, 3, 0) == MAX                   # groups of a fraction of a channel
        assert f(8, 128, 28, 28, 0, 0) == MAX
        assert f(0, 128, 28, 28, 32, 0) == MAX
        assert f(8, 128, 28, 28, 32, 0x100) == MAX
        assert f(8, 128, 28, 28, 32, B.WINO_IO_F16 | B.WINO_IO_BF16) == MAX
        assert f(2**31 - 1, 4, 1, 1, 4, 0) == MAX               # an image a workgroup, past 2^30
    assert B.wino_act8_workspace_bytes(1, 8, 4, 4, B.WINO_FLAG_RELU) == MAX
    assert B.wino_act8_workspace_bytes(2**31 - 1, 4, 1, 1, 0) == MAX
    assert B.wino_conv2d_wgrad_workspace_bytes(1, 32, 2, 56, 32, 0, 0) == MAX     # no output row
    assert B.wino_conv2d_wgrad_workspace_bytes(1, 32, 56, 56, 32, -1, 0) == MAX
    assert B.wino_conv2d_wgrad_workspace_bytes(64, 8, 8192, 8192, 8, 1, 0) == MAX  # 2^32 pixels


def _norm(x=at(1), gamma=at(2), beta=at(3), y=at(4), stats=at(5), q=at(6), N=1, C=8, H=4, W=4, G=2, eps=1e-5, flags=0,
          ws=None, wsb=0):
    return B.wino_group_norm_nhwc(x, gamma, beta, y, stats, q, N, C, H, W, G, eps, flags, ws, wsb, 0)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INV), (dict(y=None), INV), (dict(N=0), INV), (dict(C=0), INV), (dict(H=0), INV), (dict(W=-3), INV),
    (dict(G=0), INV), (dict(G=3), INV), (dict(G=16), INV), (dict(eps=-1.0), INV), (dict(eps=float("nan")), INV),
    (dict(q=at(6) + 8), INV), (dict(y=at(1)), INV), (dict(y=at(1) + 64), INV), (dict(stats=at(4)), INV),
    (dict(q=at(1)), INV), (dict(stats=at(2)), INV), (dict(N=2**31 - 1, C=2**31 - 2), INV),
    (dict(flags=0x100), UNS), (dict(flags=B.WINO_FLAG_ACT8), UNS), (dict(flags=B.WINO_FLAG_RELU | B.WINO_FLAG_SILU), UNS),
    (dict(flags=B.WINO_IO_F16 | B.WINO_IO_BF16), UNS), (dict(flags=B.WINO_PREC_F16), UNS),
    (dict(N=2**31 - 1, C=4, H=1, W=1, y=at(4) + (1 << 38)), UNS),
    (dict(C=64, H=512, W=512, G=1), WS), (dict(C=64, H=512, W=512, G=1, ws=at(9), wsb=16), WS),
])
def test_group_norm_refuses(kw, status):
    assert _norm(**kw) == status


def test_apply_refuses():
    def call(x=at(1), stats=at(5), y=at(4), G=2, flags=0, W=4):
        return B.wino_group_norm_apply_nhwc(x, stats, at(2), at(3), y, 1, 8, 4, W, G, flags, 0)
    assert call(x=None) == INV and call(stats=None) == INV and call(y=None) == INV and call(G=5) == INV
    assert call(y=at(5)) == INV and call(W=0) == INV
    assert call(x=at(1) + 4, flags=B.WINO_FLAG_ACT8) == INV
    assert call(flags=0x200) == UNS


def _back(dy=at(1), x=at(2), stats=at(3), gamma=at(4), beta=at(5), dx=at(6), dgamma=at(7), dbeta=at(8), N=1, C=8, H=4,
          W=4, G=2, flags=0, ws=at(9), wsb=1 << 20):
    return B.wino_group_norm_backward_nhwc(dy, x, stats, gamma, beta, dx, dgamma, dbeta, N, C, H, W, G, flags, ws, wsb, 0)


@pytest.mark.parametrize("kw,status", [
    (dict(dy=None), INV), (dict(x=None), INV), (dict(stats=None), INV), (dict(dx=None), INV), (dict(G=3), INV),
    (dict(H=0), INV), (dict(dx=at(1)), INV), (dict(dgamma=at(4)), INV), (dict(dbeta=at(7)), INV), (dict(dgamma=at(9)), INV),
    (dict(x=at(2) + 1, flags=B.WINO_FLAG_ACT8), INV), (dict(ws=at(9) + 2), INV), (dict(ws=None), WS), (dict(wsb=8), WS),
    (dict(flags=0x1000), UNS), (dict(flags=B.WINO_FLAG_RELU | B.WINO_FLAG_SILU), UNS), (dict(flags=B.WINO_IO_MASK), UNS),
])
def test_group_norm_backward_refuses(kw, status):
    assert _back(**kw) == status


def test_checkpoint_refuses():
    def pack(x=at(1), q=at(2), H=4, flags=0, ws=None, wsb=0, C=8):
        return B.wino_act8_pack_nhwc(x, q, 1, C, H, 4, flags, ws, wsb, 0)
    assert pack(x=None) == INV and pack(q=None) == INV and pack(q=at(2) + 4) == INV and pack(H=0) == INV
    assert pack(q=at(1)) == INV and pack(flags=B.WINO_FLAG_SILU) == UNS and pack(flags=B.WINO_IO_MASK) == UNS
    assert pack(H=1 << 20) == WS
    def unpack(q=at(2), x=at(1), H=4, flags=0):
        return B.wino_act8_unpack_nhwc(q, x, 1, 8, H, 4, flags, 0)
    assert unpack(q=None) == INV and unpack(x=None) == INV and unpack(q=at(2) + 8) == INV and unpack(H=-1) == INV
    assert unpack(x=at(2) + 32) == INV and unpack(flags=B.WINO_FLAG_ACT8) == UNS


def _wgrad(x=at(1), dy=at(2), dg=at(3), stats=at(4), gamma=at(5), beta=at(6), G=2, N=1, C=8, H=4, W=4, K=8, pad=1, flags=0,
           ws=at(7), wsb=1 << 30):
    return B.wino_conv2d_wgrad_nhwc(x, dy, dg, stats, gamma, beta, G, N, C, H, W, K, pad, flags, ws, wsb, 0)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INV), (dict(dy=None), INV), (dict(dg=None), INV), (dict(N=0), INV), (dict(C=0), INV), (dict(K=0), INV),
    (dict(pad=-1), INV), (dict(H=2, pad=0), INV), (dict(G=3), INV), (dict(G=0), INV), (dict(dg=at(1)), INV),
    (dict(dg=at(2)), INV), (dict(dg=at(7)), INV), (dict(x=at(1) + 8, flags=B.WINO_FLAG_ACT8), INV), (dict(ws=None), WS),
    (dict(wsb=64), WS), (dict(flags=0x100), UNS), (dict(stats=None, flags=B.WINO_FLAG_SILU), UNS),
    (dict(flags=B.WINO_IO_MASK), UNS), (dict(ws=at(7) + 1), INV),
])
def test_weight_gradient_refuses(kw, status):
    assert _wgrad(**kw) == status
