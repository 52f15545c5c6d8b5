"""The 64-bit reference of the 8-bit checkpoint at channels whose range is a few units
in the last place of their centre (CPU only): its codes end at 127 on both sides, where
the quotient alone would go past a byte."""
import numpy as np
import pytest

from oracle import train


@pytest.mark.parametrize("m", [1, 3, 101, 201, 253])
def test_codes_of_a_narrow_channel(m):
    x = (np.float32(1000.0) + np.arange(m + 1) * np.spacing(np.float32(1000.0))).astype(np.float32).reshape(1, 1, -1, 1)
    codes, centre, step = train.act8_pack(x)
    quotient = (x - centre[:, None, None]) * (np.float32(127.0) / (np.float32(127.0) * step[:, None, None]))
    assert np.abs(quotient).max() > 127.0
    assert codes.min() >= -127 and codes.max() <= 127
    # the centre's rounding is half a unit, the code's half a step, the sum has none in 64 bits
    v = train.act8_unpack(codes, centre, step)
    assert (np.abs(v - x) <= 0.5 * step + 0.5 * np.spacing(np.float32(1000.0)) + m * np.spacing(x) * 2.0 ** -22).all()
