"""Scales whose product with log2 e, which the exponents take, is past fp32's range (CPU only)."""
import pytest
import torch

from paper_1903_01521_amd import binding as B
from test_block_abi_cpu import INV, _attn, _attn_back


@pytest.mark.parametrize("scale,refused", [(3.4e38, True), (2.36e38, True), (2.35e38, False), (2.0 ** -149, False)])
def test_largest_scale(scale, refused):
    if refused:
        assert _attn(scale=scale) == INV and _attn_back(scale=scale) == INV
    elif not torch.cuda.is_available():               # what follows the checks does not run: no device here
        assert _attn(scale=scale) == B.WINO_ERR_HIP and _attn_back(scale=scale) == B.WINO_ERR_HIP
