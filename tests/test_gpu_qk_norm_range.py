"""The norm of vectors whose squares are past fp32's range, at both ends, beside others that are not."""
import numpy as np
import pytest

import test_gpu_qk_norm as qk_norm
from test_gpu_qk_norm import call, check_backward, check_forward, make
from train_helpers import rounded

pytestmark = pytest.mark.gpu

# teams of 2 to 64 lanes
SIZES = [(2, 9, 7, 3, 2, 64, 32), (1, 5, 6, 2, 1, 128, 128), (3, 4, 5, 2, 2, 7, 4), (1, 30, 2, 5, 1, 24, 8), (2, 3, 3, 2, 2, 97, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("log2,eps", [(100, 1e-6), (66, 0.0), (63, 1e30), (-66, 0.0), (-100, 0.0), (-66, 2.0 ** -130), (-100, 2.0 ** -149)])
def test_vectors_past_the_range_of_squares(size, log2, eps, dtype, monkeypatch):
    monkeypatch.setattr(qk_norm, "EPS", float(np.float32(eps)))
    d = make(size, dtype, 111, 0)
    rng = np.random.default_rng(112)
    for x in "qk":
        # a third of the heads as they are; where eps is 0 they need none
        up = np.where(rng.random(d[x].shape[:3]) < 0.67, 2.0 ** log2, 1.0)
        d[x] = rounded(d[x] * up[..., None], dtype)
    check_forward(d, size, dtype, call(d, size, dtype), False)
    check_backward(d, size, dtype, call(d, size, dtype, back=True), False)


def test_zeros_and_the_largest_values(monkeypatch):
    size = (1, 6, 4, 2, 1, 64, 32)
    d = make(size, "f32", 113, 0)
    d["q"][0, 0], d["q"][0, 1] = 0.0, 3.4e38
    d["q"][0, 2], d["q"][0, 3] = np.float32(2.0 ** -149), -3.4e38
    d["q"][0, 3, 1, 5:] = 0.0
    check_forward(d, size, "f32", call(d, size, "f32"), False)
    monkeypatch.setattr(qk_norm, "EPS", 0.0)
    d["q"][0, 0] = 1.0                                      # 0 / 0 by the definition
    check_forward(d, size, "f32", call(d, size, "f32"), False)
