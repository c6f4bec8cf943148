"""The gradient of log probabilities where its factors, or their products with the scale, come to the end of fp32: places
without probability give 0, others what the formula gives as long as that is a number of the type."""
import numpy as np
import pytest
import torch

from oracle import learn_oracle as L
from paper_2309_06973_amd.q8 import Q8
from test_gpu_log_probs import check_grad, make, near

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF = float("inf")


@pytest.fixture(scope="module")
def ops():
    o = Q8()
    yield o
    torch.cuda.synchronize()
    o.close()


def setup(cols, low, scale):
    """Rows whose z are of order 1 whatever the scale is, every third place without probability."""
    x, t = make(5, cols, torch.float32, 3) / scale, torch.tensor([0, -1, 2, 3, 6], device=DEV)
    x[:, 1::3] = low
    ref = L.Logs(x, scale)
    norm, h = (torch.from_numpy(v).float().to(DEV) for v in (ref.norm, ref.entropy))
    return x, t, ref, norm, h


@pytest.mark.parametrize("low", [-INF, torch.finfo(torch.float32).min])
@pytest.mark.parametrize("cols", [100, 900, 3000, 20000])
def test_large_factors(ops, cols, low):
    """Sizes that stay below 3e38 for p (log p + H) up to 8 with the scale, and above it without p."""
    full = lambda *v: torch.tensor(v, device=DEV)
    for scale, size in ((1.0, 1e37), (2.0 ** 40, 1e25), (2.0 ** 64, 1e17), (1.0, 3e37)):
        x, t, ref, norm, h = setup(cols, low, scale)
        for some in (dict(g_logp=full(-3.0, 1.0, 0.0, 2.0, 1.0), g_entropy=full(size, -size, size / 2, 1e4, -size)),
                     dict(g_logp=full(size, 1.0, -size, 2.0, size), g_entropy=None),
                     dict(g_logp=full(size, 1.0, -size, 2.0, size), g_lse=full(-size, size, 1.0, -size, size), g_entropy=full(size, size, -size, 0.0, 1.0))):
            print(f"large factors cols={cols} low={low} scale={scale} size={size} {list(some)}", flush=True)
            got = ops.log_probs_grad(x, t, norm, entropy=h, scale=scale, **some)
            check_grad(got, ref, torch.float32, t, **some)
            assert (got[:, 1::3] == 0).all()


@pytest.mark.parametrize("cols", [100, 900, 3000])
def test_products_with_the_scale_beyond_fp32(ops, cols):
    """The target's own place is infinite, as the formula's value is beyond fp32; the others' products are not, where p is small enough."""
    scale = 2.0 ** 64
    x, t, ref, norm, h = setup(cols, -INF, scale)
    got = ops.log_probs_grad(x, t, norm, g_logp=torch.full((5,), 1e25, device=DEV), scale=scale)
    assert (got[:, 1::3] == 0).all() and not torch.isnan(got).any()
    assert (got[1] == 0).all() and got[0, 0] == INF and (got[0, 3::3] <= 0).all()


@pytest.mark.parametrize("cols", [100, 900, 3000])
def test_factors_whose_difference_is_beyond_fp32(ops, cols):
    for scale in (1.0, 0.25):
        x, t, ref, norm, h = setup(cols, -INF, scale)
        big = torch.tensor([3e38, -3e38, 3e38, -2e38, 1e38], device=DEV)
        for some in (dict(g_logp=big, g_lse=-big), dict(g_logp=big, g_lse=-big, g_entropy=big / 16)):
            got = ops.log_probs_grad(x, t, norm, entropy=h, scale=scale, **some)
            assert (got[:, 1::3] == 0).all()
            # one place of a row is -4e38 by the formula (p 0.68 or 0.66 of -6e38): infinite in fp32
            want, off = ref.grad(t, **some)
            beyond = np.abs(want) > 3.41e38
            assert beyond.sum() == (scale == 1.0 and cols != 900)
            want[beyond] = np.copysign(np.inf, want[beyond])
            near(got, want, off + L.U * np.abs(want), "grad")


@pytest.mark.parametrize("scale", [2.0 ** -100, 1e-38])
def test_factors_that_the_scale_takes_below_fp32(ops, scale):
    """g scale is no number of fp32 here; a row that holds NaN is NaN all the same, as its factor is not 0."""
    x = torch.full((2, 300), 3.0, device=DEV)
    x[0, 7] = float("nan")
    t = torch.tensor([1, 1], device=DEV)
    r = ops.log_probs(x, t, scale=scale)
    got = ops.log_probs_grad(x, t, r.norm, g_logp=torch.full((2,), 1e-20, device=DEV), scale=scale)
    assert torch.isnan(got[0]).all() and (got[1] == 0).all()
