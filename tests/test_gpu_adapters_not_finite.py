"""Adapters and rows that are not finite: what they give stays in their rows, and nothing of it comes out as a number."""
import pytest
import torch

from paper_2309_06973_amd.q8 import Q8
from test_gpu_adapters import DTYPES, setup

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ops():
    o = Q8()
    yield o
    torch.cuda.synchronize()
    o.close()


def test_what_is_not_finite_stays_in_its_rows(ops):
    """Row by row against the clean result; an adapter's NaN, an infinity in B, in x, and rows that name no adapter."""
    for m in (40, 400):
        for dtype in DTYPES:
            y, x, _, a, b, num, _ = setup(ops, m, 200, 152, 20, 9, dtype, "random")
            num[5], num[6], num[7], num[8], num[9] = 9, 1 << 40, -(1 << 60), 1, 1
            clean = ops.adapters(y, x, a, b, num)
            a[2], b[4, 3] = NAN, INF
            x[8], x[9, 17] = NAN, INF
            got = ops.adapters(y, x, a, b, num)
            all_nan = (num == 2) | (num >= 9)
            all_nan[8] = True
            want = clean.clone()
            want[all_nan] = NAN
            four = num == 4
            assert not torch.isfinite(got[four][:, 3]).any() and not torch.isfinite(got[9]).any()
            want[9] = got[9]
            want[four, 3] = got[four, 3]
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [7, 300])
def test_sums_that_overflow(ops, m, dtype):
    """Where scale x A' is beyond fp32: infinite or NaN, as B goes, in all columns of B that are not 0."""
    y, x, _, a, b, num, scale = setup(ops, m, 70, 64, 5, 2, dtype, "one")
    b[:] = b.abs() + 0.25
    x[3] = 4.0
    a[:] = a.abs() + 0.5
    scale[:] = 3e38
    out = ops.adapters(y.float(), x, a, b, num, scale=scale)
    assert not torch.isfinite(out[3]).any()
