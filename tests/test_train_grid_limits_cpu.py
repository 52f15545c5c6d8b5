"""Launches of 2^32 threads, which the runtime refuses, are refused by the checks before
anything is enqueued (CPU only: no call here reaches a kernel)."""
from paper_1903_01521_amd import binding as B

FAKE = 0x100000000                     # never dereferenced: every call here is refused
MAX = 2**64 - 1


def test_weight_gradients_of_too_many_filters_and_channels():
    # 8 channels by 32 filters by a row of taps take 256 threads of the last launch
    for C, K in ((40000, 40000), (1 << 20, 1700)):
        assert -(-C // 8) * -(-K // 32) * 3 * 256 >= 2**32
        assert B.wino_conv2d_wgrad_workspace_bytes(1, C, 4, 4, K, 1, 0) == MAX
        assert B.wino_conv2d_wgrad_nhwc(FAKE, FAKE << 8, FAKE << 16, None, None, None, 0, 1, C, 4, 4, K, 1, 0, FAKE << 20,
                                        1 << 50, 0) == B.WINO_ERR_UNSUPPORTED
    C, K = 36864, 32768                # just below
    assert -(-C // 8) * -(-K // 32) * 3 * 256 < 2**32
    assert B.wino_conv2d_wgrad_workspace_bytes(1, C, 4, 4, K, 1, 0) < MAX
