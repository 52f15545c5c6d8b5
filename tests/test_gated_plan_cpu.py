"""The gated layer's plan: what the query answers, and that the sizes of the tiles' tests reach
every shape that a plan can name, whole and in parts (host only)."""
import pytest

from gated_sizes import NARROW, ODD, SIZES, SMALL, SQUARE, WIDE, plan
from paper_1903_01521_amd import binding as B

F32, F16, BF16 = 0, B.WINO_IO_F16, B.WINO_IO_BF16


@pytest.mark.parametrize("flags", [F32, F16, BF16])
def test_sizes_reach_every_shape(flags):
    shapes = [SQUARE, NARROW, SMALL] if flags == F32 else [WIDE, SQUARE, NARROW, SMALL]
    seen = [set(), set(), set()]
    for size in SIZES:
        results, parts = plan(size, flags)
        for s, r, p in zip(seen, results, parts):
            s.add((r, p > 1))
        assert plan(size, flags, False)[0][0] == results[0]
    # a unit's gate and value are to be in one wave: no small tiles, and its sum is whole
    assert seen[0] >= {(s, False) for s in shapes if s != SMALL}
    assert seen[1] == {(s, p) for s in shapes for p in (False, True)}
    # dw of wide tiles in one part is of 2^19 results and few tokens, where they are no gain
    assert seen[2] >= {(s, True) for s in shapes} | {(s, False) for s in shapes if s in (SQUARE, NARROW)}
    odd = {plan(size, flags)[0][0] for size in ODD}
    assert odd >= set(shapes[:-1])


def test_few_tokens():
    for M in (1, 8):
        assert plan((M, 64, 96), BF16, False) == ((0, 0, 0), (1, 0, 0))
        assert plan((M, 64, 96), BF16)[0][0] == NARROW
    assert plan((9, 64, 96), BF16, False) == ((NARROW, 0, 0), (1, 0, 0))


def test_parts_fit_the_workspace():
    for size in SIZES:
        M, C, K = size
        for flags, each in ((F32, 4), (BF16, 2)):
            _, parts = plan(size, flags)
            need = B.wino_gated_layer_backward_workspace_bytes(1, C, 1, M, K, flags)
            sums = sum(p * n * 4 for p, n in ((parts[1], M * C), (parts[2], 2 * K * C)) if p > 1)
            assert need >= sums + 2 * M * K * each


@pytest.mark.parametrize("kw,status", [
    (dict(C=0), B.WINO_ERR_INVALID_ARG), (dict(K=-1), B.WINO_ERR_INVALID_ARG), (dict(N=2**30, H=2**20), B.WINO_ERR_INVALID_ARG),
    (dict(flags=B.WINO_IO_MASK), B.WINO_ERR_UNSUPPORTED), (dict(flags=B.WINO_FLAG_PAIRS), B.WINO_ERR_UNSUPPORTED),
    (dict(flags=B.WINO_FLAG_RELU | B.WINO_FLAG_SILU), B.WINO_ERR_UNSUPPORTED), (dict(K=2**30, C=2), B.WINO_ERR_UNSUPPORTED),
])
def test_refusals(kw, status):
    a = dict(N=1, C=8, H=1, W=1, K=8, flags=0)
    a.update(kw)
    for backward in (False, True):
        assert B.wino_gated_layer_plan(*a.values(), backward)[0] == status
    assert B.lib().wino_gated_layer_plan(1, 8, 1, 1, 8, 0, 0, None, None) == B.WINO_ERR_INVALID_ARG
