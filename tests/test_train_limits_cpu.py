"""Channel counts at the limit of 32-bit channel numbers: a workgroup's last column lies up
to 1024 channels past the first, so the norm and the checkpoint take at most 2^30 (CPU
only: no call here reaches a kernel)."""
import pytest

from paper_1903_01521_amd import binding as B

FAKE = 0x100000000                     # never dereferenced: every call here is refused
MAX, TOP = 2**64 - 1, 2**30


def at(i):
    return FAKE + (i << 42)


@pytest.mark.parametrize("C", [TOP + 4, 2**31 - 1])
def test_more_channels_are_refused(C):
    G = 4 if C % 4 == 0 else 1
    assert B.wino_group_norm_workspace_bytes(1, C, 1, 1, G, 0) == MAX
    assert B.wino_group_norm_backward_workspace_bytes(1, C, 1, 1, G, 0) == MAX
    assert B.wino_act8_workspace_bytes(1, C, 1, 1, 0) == MAX
    assert B.wino_act8_bytes(1, C, 1, 1) == 0
    ws, wsb = at(9), 1 << 41
    uns = B.WINO_ERR_UNSUPPORTED
    assert B.wino_group_norm_nhwc(at(1), at(2), at(3), at(4), at(5), at(6), 1, C, 1, 1, G, 1e-5, 0, ws, wsb, 0) == uns
    assert B.wino_group_norm_apply_nhwc(at(1), at(2), at(3), at(4), at(5), 1, C, 1, 1, G, 0, 0) == uns
    assert B.wino_group_norm_backward_nhwc(at(1), at(2), at(3), at(4), at(5), at(6), at(7), at(8), 1, C, 1, 1, G, 0, ws,
                                           wsb, 0) == uns
    assert B.wino_act8_pack_nhwc(at(1), at(2), 1, C, 1, 1, 0, ws, wsb, 0) == uns
    assert B.wino_act8_unpack_nhwc(at(1), at(2), 1, C, 1, 1, 0, 0) == uns


def test_the_limit_itself_is_taken():
    # parts and a row of statistics of some workgroups' columns: a size, far below the limit's 2^64 - 1
    assert 0 < B.wino_group_norm_workspace_bytes(1, TOP, 1, 1, 1, 0) < 2**40
    assert B.wino_act8_bytes(1, TOP, 1, 1) == TOP + TOP * 8


def test_many_images_of_many_groups():
    # four channels a workgroup would be 2^31 of them: sixteen are taken, which fit the limit,
    # and need no workspace
    assert B.wino_group_norm_workspace_bytes(2**24, 512, 1, 1, 128, 0) == 0
