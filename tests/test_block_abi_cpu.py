"""Sizes and refusals of the attention half's calls: arguments are checked before any HIP
call (CPU only: no call here reaches a kernel)."""
import pytest
import torch

from paper_1903_01521_amd import binding as B

FAKE = 0x100000000                     # never dereferenced: every call here is refused
MAX = 2**64 - 1
INV, UNS, WS = B.WINO_ERR_INVALID_ARG, B.WINO_ERR_UNSUPPORTED, B.WINO_ERR_WORKSPACE
NAN, INF = float("nan"), float("inf")


def at(i):
    return FAKE + (i << 40)


def _norm(q=at(1), k=at(2), gq=at(3), gk=at(4), rot=at(5), qpos=at(6), kpos=at(7), yq=at(8), yk=at(9), N=2, Lq=5, Lk=7,
          Hq=4, Hk=2, D=64, R=32, T=100, ldq=256, ldk=128, eps=1e-6, flags=0):
    return B.wino_qk_norm_nhwc(q, k, gq, gk, rot, qpos, kpos, yq, yk, N, Lq, Lk, Hq, Hk, D, R, T, ldq, ldk, eps, flags, 0)


BAD_NORM = [
    (dict(q=None), INV), (dict(N=0), INV), (dict(Lq=0), INV), (dict(Lk=-1), INV), (dict(Hq=0), INV), (dict(Hk=0), INV),
    (dict(D=0), INV), (dict(ldq=255), INV), (dict(ldk=64), INV), (dict(R=-2), INV), (dict(R=33), INV), (dict(R=66), INV),
    (dict(rot=None), INV), (dict(T=0), INV), (dict(qpos=None, T=4), INV), (dict(kpos=None, T=6), INV), (dict(eps=-1.0), INV),
    (dict(eps=NAN), INV), (dict(N=2**31 - 1, Lq=2**31 - 1), INV), (dict(T=2**31 - 1, R=64, D=64), None),
    (dict(D=130, ldq=520, ldk=260), UNS), (dict(flags=B.WINO_FLAG_SILU), UNS), (dict(flags=B.WINO_IO_MASK), UNS),
    (dict(flags=0x100), UNS), (dict(N=2**20, Lq=2**11, ldq=256, qpos=None, T=2**11), None),
]


@pytest.mark.parametrize("kw,status", [b for b in BAD_NORM if b[1] is not None] + [
    (dict(yq=None), INV), (dict(yk=None), INV), (dict(yq=at(1)), INV), (dict(yk=at(8) + 64), INV), (dict(yq=at(5)), INV),
    (dict(yk=at(7)), INV), (dict(yk=at(4)), INV),
    # 2^31 tokens and more
    (dict(N=2**11, Lq=2**20, Hq=1, D=2, R=0, ldq=2, Lk=1, Hk=1, ldk=2), UNS),
])
def test_norm_refuses(kw, status):
    assert _norm(**kw) == status


def _norm_back(dyq=at(10), dyk=at(11), dq=at(12), dk=at(13), dgq=at(14), dgk=at(15), ws=at(16), wsb=1 << 30, q=at(1),
               k=at(2), gq=at(3), gk=at(4), rot=at(5), qpos=at(6), kpos=at(7), N=2, Lq=5, Lk=7, Hq=4, Hk=2, D=64, R=32,
               T=100, ldq=256, ldk=128, eps=1e-6, flags=0):
    return B.wino_qk_norm_backward_nhwc(dyq, dyk, q, k, gq, gk, rot, qpos, kpos, dq, dk, dgq, dgk, N, Lq, Lk, Hq, Hk, D,
                                        R, T, ldq, ldk, eps, flags, ws, wsb, 0)


@pytest.mark.parametrize("kw,status", [b for b in BAD_NORM if b[1] is not None] + [
    (dict(dyq=None), INV), (dict(dyk=None), INV), (dict(dq=None), INV), (dict(dk=None), INV), (dict(dq=at(1)), INV),
    (dict(dk=at(11)), INV), (dict(dgq=at(14), dgk=at(14)), INV), (dict(dgq=at(3)), INV), (dict(ws=at(14)), INV),
    (dict(ws=None), WS), (dict(wsb=64), WS), (dict(ws=at(16) + 8), INV),
    # rows of one stride that do and do not lie between each other: the second ends at a workspace too small
    (dict(ldq=384, ldk=384, dk=at(12) + 255 * 4), INV), (dict(ldq=384, ldk=384, dk=at(12) + 257 * 4), INV),
    (dict(ldq=384, ldk=384, dk=at(12) - 127 * 4), INV), (dict(ldq=384, ldk=392, dk=at(12) + 256 * 4), INV),
])
def test_norm_backward_refuses(kw, status):
    assert _norm_back(**kw) == status


def test_interleaved_rows_do_not_overlap():
    # what follows the check of overlaps does not run: no device here
    if not torch.cuda.is_available():
        assert _norm_back(ldq=384, ldk=384, dk=at(12) + 256 * 4) == B.WINO_ERR_HIP
        assert _norm_back(ldq=384, ldk=384, dk=at(12) - 128 * 4) == B.WINO_ERR_HIP


def test_norm_workspace_bytes():
    f = B.wino_qk_norm_backward_workspace_bytes
    assert f(2, 5, 7, 4, 2, 64, 0) >= 2 * 64 * 4 and f(2, 5, 0, 4, 0, 64, 0) >= 64 * 4
    assert f(64, 3136, 3136, 4, 4, 64, B.WINO_IO_BF16) <= 2048 * 64 * 4 + 16
    for bad in ((0, 5, 7, 4, 2, 64, 0), (2, 0, 7, 4, 2, 64, 0), (2, 5, 7, 4, 0, 64, 0), (2, 5, 0, 4, 2, 64, 0),
                (2, 5, 7, 4, 2, 129, 0), (2, 5, 7, 4, 2, 64, 0x100), (2, 5, 7, 2**25, 2, 128, 0), (2, 5, 7, 4, 2, 0, 0),
                (2, 5, 7, 4, 2, 64, B.WINO_IO_MASK), (2**20, 2**11, 1, 1, 1, 2, 0)):
        assert f(*bad) == MAX


def _attn(q=at(1), k=at(2), v=at(3), klen=at(4), mask=at(5), y=at(6), lse=at(7), N=2, Lq=50, Lk=70, Hq=4, Hk=2, D=64, ldq=256,
          ldk=128, ldv=128, scale=0.125, flags=0, ws=at(8), wsb=1 << 30):
    return B.wino_cross_attention_nhwc(q, k, v, klen, mask, y, lse, N, Lq, Lk, Hq, Hk, D, ldq, ldk, ldv, scale, flags, ws,
                                       wsb, 0)


BAD_ATTN = [
    (dict(q=None), INV), (dict(k=None), INV), (dict(v=None), INV), (dict(N=0), INV), (dict(Lq=0), INV), (dict(Lk=0), INV),
    (dict(Hq=0), INV), (dict(Hk=0), INV), (dict(Hk=3, ldk=192, ldv=192), INV), (dict(Hq=1, ldq=64), INV), (dict(D=-1), INV),
    (dict(ldq=255), INV), (dict(ldk=127), INV), (dict(ldv=1), INV), (dict(scale=0.0), INV), (dict(scale=-0.1), INV),
    (dict(scale=NAN), INV), (dict(scale=INF), INV), (dict(N=2**31 - 1, Lq=2**31 - 1), INV),
    (dict(D=136, ldq=544, ldk=272, ldv=272), UNS), (dict(flags=B.WINO_FLAG_RELU), UNS), (dict(flags=B.WINO_FLAG_PAIRS), UNS),
    (dict(flags=B.WINO_IO_MASK), UNS), (dict(flags=0x200), UNS), (dict(ws=at(8) + 4), INV),
    # a pair's rows past 2^31
    (dict(N=1, Lq=2**30, Hq=4, Hk=1, D=1, ldq=4, Lk=1, ldk=1, ldv=1, y=at(6) + (1 << 39)), UNS),
    # workgroups past 2^30
    (dict(N=2**29, Lq=1, Hq=4, Hk=4, D=1, ldq=4, Lk=1, ldk=4, ldv=4, y=at(6) + (1 << 39)), UNS),
]


@pytest.mark.parametrize("kw,status", BAD_ATTN + [
    (dict(y=None), INV), (dict(y=at(1)), INV), (dict(y=at(2) + 4), INV), (dict(y=at(3)), INV), (dict(lse=at(6)), INV),
    (dict(lse=at(4)), INV), (dict(y=at(5)), INV), (dict(Lq=1, Lk=5000, ws=None), WS), (dict(Lq=1, Lk=5000, wsb=1000), WS),
    (dict(Lq=1, Lk=5000, ws=at(2)), INV),
])
def test_attention_refuses(kw, status):
    assert _attn(**kw) == status


def _attn_back(dy=at(9), q=at(1), k=at(2), v=at(3), y=at(6), lse=at(7), klen=at(4), mask=at(5), dq=at(10), dk=at(11),
               dv=at(12), N=2, Lq=50, Lk=70, Hq=4, Hk=2, D=64, ldq=256, ldk=128, ldv=128, scale=0.125, flags=0, ws=at(8),
               wsb=1 << 30):
    return B.wino_cross_attention_backward_nhwc(dy, q, k, v, y, lse, klen, mask, dq, dk, dv, N, Lq, Lk, Hq, Hk, D, ldq,
                                                ldk, ldv, scale, flags, ws, wsb, 0)


@pytest.mark.parametrize("kw,status", BAD_ATTN + [
    (dict(dy=None), INV), (dict(y=None), INV), (dict(lse=None), INV), (dict(dq=None), INV), (dict(dk=None), INV),
    (dict(dv=None), INV), (dict(dq=at(1)), INV), (dict(dk=at(2)), INV), (dict(dv=at(11)), INV), (dict(dq=at(9)), INV),
    (dict(dq=at(7)), INV), (dict(dk=at(8)), INV), (dict(ws=None), WS), (dict(wsb=2 * 4 * 50 * 4 - 1), WS),
])
def test_attention_backward_refuses(kw, status):
    assert _attn_back(**kw) == status


def test_attention_workspace_bytes():
    f, b = B.wino_cross_attention_workspace_bytes, B.wino_cross_attention_backward_workspace_bytes
    assert f(16, 3136, 2048, 8, 8, 64, 0) == 0                       # rows fill the card
    assert f(1, 1, 5000, 8, 8, 64, 0) > 0                            # one token: keys in parts
    assert b(2, 50, 70, 4, 2, 64, 0) >= 2 * 4 * 50 * 4
    for bad in ((0, 5, 7, 4, 2, 64, 0), (2, 5, 7, 4, 3, 64, 0), (2, 5, 7, 4, 2, 129, 0), (2, 5, 7, 4, 2, 64, 1),
                (2, 5, 7, 2**25, 2**25, 128, 0), (2, 5, -7, 4, 2, 64, 0), (2, 5, 7, 4, 2, 64, B.WINO_IO_MASK),
                (1, 2**30, 1, 4, 1, 1, 0)):
        assert f(*bad) == MAX and b(*bad) == MAX


def _gated(x=at(1), w=at(2), bias=at(3), y=at(4), N=2, C=64, H=5, W=6, K=96, flags=0, ws=None, wsb=0):
    return B.wino_gated_layer_nhwc(x, w, bias, y, N, C, H, W, K, flags, ws, wsb, 0)


def _gated_back(dy=at(5), x=at(1), w=at(2), bias=at(3), dx=at(6), dw=at(7), dbias=at(8), N=2, C=64, H=5, W=6, K=96, flags=0,
                ws=at(9), wsb=1 << 40):
    return B.wino_gated_layer_backward_nhwc(dy, x, w, bias, dx, dw, dbias, N, C, H, W, K, flags, ws, wsb, 0)


BAD_GATED = [
    (dict(x=None), INV), (dict(w=None), INV), (dict(N=0), INV), (dict(C=0), INV), (dict(H=-2), INV), (dict(W=0), INV),
    (dict(K=0), INV), (dict(N=2**31 - 1, H=2**31 - 1), INV), (dict(flags=B.WINO_FLAG_ACT8), UNS),
    (dict(flags=B.WINO_FLAG_RELU | B.WINO_FLAG_SILU), UNS), (dict(flags=B.WINO_IO_MASK), UNS), (dict(flags=0x400), UNS),
    (dict(N=2**11, C=1, H=2**10, W=2**10, K=1), UNS), (dict(N=1, C=1, H=1, W=1, K=2**30), UNS), (dict(ws=at(9) + 8), INV),
]


@pytest.mark.parametrize("kw,status", BAD_GATED + [
    (dict(y=None), INV), (dict(y=at(1)), INV), (dict(y=at(2)), INV), (dict(y=at(3)), INV),
])
def test_gated_refuses(kw, status):
    assert _gated(**kw) == status


@pytest.mark.parametrize("kw,status", BAD_GATED + [
    (dict(dy=None), INV), (dict(dx=None, dw=None, dbias=None), INV), (dict(dx=at(1)), INV), (dict(dw=at(2)), INV),
    (dict(dbias=at(3)), INV), (dict(dx=at(5)), INV), (dict(dw=at(6)), INV), (dict(dx=at(9)), INV), (dict(ws=None), WS),
    (dict(wsb=64), WS),
])
def test_gated_backward_refuses(kw, status):
    assert _gated_back(**kw) == status


def test_launches_of_2_to_the_32_threads_are_refused():
    """256 threads a workgroup: fewer than 2^24 workgroups a launch."""
    assert _attn(N=2**24, Lq=1, Lk=1, Hq=1, Hk=1, D=1, ldq=1, ldk=1, ldv=1) == UNS               # a token's workgroup each
    assert B.wino_cross_attention_workspace_bytes(2**24, 1, 1, 1, 1, 1, 0) == MAX
    assert B.wino_cross_attention_workspace_bytes(2**24 - 8, 1, 1, 1, 1, 1, 0) == 0
    assert B.wino_cross_attention_backward_workspace_bytes(2**23, 1, 65, 2, 2, 1, 0) == MAX      # two workgroups' keys
    f, b = B.wino_gated_layer_workspace_bytes, B.wino_gated_layer_backward_workspace_bytes
    assert f(1, 1, 1, 1, 2**26, 0) == MAX and f(1, 1, 1, 1, 2**26 - 64, 0) == 0                  # a wave for each unit
    assert f(2**14, 1, 2**8, 2**8, 2**9, 0) == MAX and f(2**12, 1, 2**8, 2**8, 2**8, 0) == 0     # tiles
    assert b(2**14, 1, 2**8, 2**8, 2**9, 0) == MAX
    # 4 tokens a workgroup where heads are of 127
    assert _norm(N=2**26, Lq=1, Lk=1, Hq=1, Hk=1, D=127, R=0, ldq=127, ldk=127) == UNS


def test_gated_workspace_bytes():
    f, b = B.wino_gated_layer_workspace_bytes, B.wino_gated_layer_backward_workspace_bytes
    assert f(32, 512, 14, 14, 2048, B.WINO_IO_BF16) == 0
    assert b(2, 64, 5, 6, 96, B.WINO_IO_BF16) >= 2 * 5 * 6 * 2 * 96 * 2
    for bad in ((0, 64, 5, 6, 96, 0), (2, 64, 5, 6, 0, 0), (2, 64, 5, 6, 96, 0x100), (2, 64, 5, 6, 96, B.WINO_FLAG_PAIRS),
                (2**11, 1, 2**10, 2**10, 1, 0), (2**31 - 1, 64, 2**31 - 1, 6, 96, 0)):
        assert f(*bad) == MAX and b(*bad) == MAX


def test_binding_checks_tensors():
    t = torch.empty(2, 3, 4, 5)
    with pytest.raises(ValueError):
        B._rows(t, torch.float32, 3, 5, 20)                                            # not on a GPU
    with pytest.raises(ValueError):
        B._rows(t.transpose(1, 2), torch.float32, 4, 5, 20)                            # heads are not together
    with pytest.raises(ValueError):
        B._rows(t[:, :, :2], torch.float32, 3, 5, 10)                                  # tokens are 20 apart
    B._check_rows(t, 20)
    B._check_rows(t[:, :, :2], 20)
    B._check_rows(t[:1, :1], 999)                                    # one token: any distance
    B._check_rows(t.view(-1), 999)                                   # sizes are the call's
    for bad, ld in ((t.transpose(1, 2), 20), (t[:, :, :2], 10), (t, 21), (t[:, ::2], 20), (t.view(-1)[::2], 20)):
        with pytest.raises(ValueError):
            B._check_rows(bad, ld)
    with pytest.raises(ValueError):
        B._iptr(torch.empty(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        B._mptr(torch.empty(3))
