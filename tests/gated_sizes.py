"""Sizes of the gated layer that reach every tile shape, whole and in parts: tokens, channels
and units beside the tiles' edges, no tile's multiple but where it is said."""
from paper_1903_01521_amd import binding as B

WIDE, SQUARE, NARROW, SMALL = 128 * 256, 128 * 128, 64 * 128, 64 * 64

# tokens M, channels C, units K; the products that a row is there for (16-bit types | fp32)
SIZES = [
    (16640, 24, 1000),       # first wide, one step of 32 channels | square; dx in parts
    (16643, 40, 1000),       # two steps
    (16901, 72, 872),        # three steps; dx square in parts
    (16897, 136, 1000),      # five steps
    (58347, 16, 72),         # units that end inside a wide tile's second half
    (6275, 512, 2056),       # first square: a whole number of steps | dw square
    (50401, 72, 24),         # dx square, whole
    (56185, 136, 24),        # dx wide, whole
    (35111, 72, 1392),       # dx wide in parts, dw square in parts
    (3825, 976, 2064),       # dw wide in parts
    (67, 1744, 1800),        # dw square, whole
    (67, 1432, 2208),        # the same of fp32
    (17827, 72, 464),        # | square in parts everywhere
    (65, 728, 1360),         # dw narrow, whole
    (2223, 16, 2736),        # dw narrow in parts, dx small in parts
    (32925, 16, 24),         # dx narrow, whole
    (11187, 16, 392),        # | dx narrow in parts
    (6271, 16, 896),         # dx narrow in parts
    (70, 24, 40),            # small, whole
]
# widths that are no whole words, so that no tile goes straight to LDS
ODD = [(16641, 27, 1001), (16641, 71, 999), (6273, 511, 2050), (50399, 67, 23), (56173, 129, 21), (17823, 73, 465)]


def plan(size, flags, backward=True):
    M, C, K = size
    status, results, parts = B.wino_gated_layer_plan(1, C, 1, M, K, flags, backward)
    assert status == B.WINO_OK
    return results, parts
