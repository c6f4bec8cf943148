"""The ends of the numbers in the 8-bit operators: rows as large as numbers get, read back."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as Q
from paper_2309_06973_amd.q8 import Q8

pytestmark = pytest.mark.gpu
DEV = "cuda"
MOST = torch.finfo(torch.float32).max


@pytest.fixture(scope="module")
def ops():
    o = Q8()
    yield o
    torch.cuda.synchronize()
    o.close()


@pytest.mark.parametrize("cols", [1, 64, 700, 3000, 9000, 40000])
def test_the_largest_numbers_come_back(ops, cols):
    """A row's largest value is read back to within the scale's step (1 / 2^23 of it) and the product's rounding, and is a
    number: that is 1.5 steps."""
    below = float(np.nextafter(np.float32(MOST), np.float32(0)))
    x = torch.zeros(5, cols, device=DEV)
    x[:, cols // 2] = torch.tensor([MOST, -MOST, below, MOST * 0.99999, float(torch.finfo(torch.bfloat16).max)], device=DEV)
    y = ops.dequantize(ops.quantize(x))
    assert torch.isfinite(y).all()
    assert ((y.double() - x.double()).abs() <= 3 * Q.U32 * x.abs().double()).all()
    # behind a norm of a single column, whose root mean square is 1: the weight itself
    h = torch.ones(1, 1, device=DEV)
    for top in (MOST, below):
        m, _ = ops.rms_norm(h, torch.full((1,), top, device=DEV), 0.0)
        assert abs(float(ops.dequantize(m).double()) / top - 1.0) <= 3 * Q.U32
