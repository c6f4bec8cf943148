"""Log probabilities and their gradient with scales that bring logits of any distance within reach of each other.  How far
numbers may be off is derived in oracle.learn_oracle; distances in another unit, a power of two, add less than 2^-148 to an exponent."""
import numpy as np
import pytest
import torch

from oracle import learn_oracle as L
from paper_2309_06973_amd.q8 import Q8, target_log_probs
from test_gpu_log_probs import check, check_grad

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF = float("inf")


@pytest.fixture(scope="module")
def ops():
    o = Q8()
    yield o
    torch.cuda.synchronize()
    o.close()


def far(rows, cols, dtype, seed):
    """Logits all over the range of the type, masked places and its ends among them."""
    x = torch.rand(rows, cols, generator=torch.Generator().manual_seed(seed)) * 2 - 1
    x = (x.double() * 3.3e38).to(dtype).to(DEV)
    x[:, 0], x[:, -1] = torch.finfo(dtype).max, torch.finfo(dtype).min
    if cols > 4:
        x[0, 2::3] = -INF
    return x


SCALES = [1e-38, 2.0 ** -126, 2.0 ** -140, 2.0 ** -149, 1e-37, 2.0 ** -100, 2.0 ** -65, float(np.nextafter(np.float32(2.0 ** -64), np.float32(0))), 2.0 ** -64, 2.0 ** -20]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [2, 7, 200, 1000, 5000, 50001])
def test_small_scales(ops, cols, dtype):
    x, t = far(6, cols, dtype, cols), torch.tensor([0, cols - 1, 1, cols // 2, -1, cols - 1], device=DEV)
    top = min(cols, 20)
    g = torch.randn(3, 6, generator=torch.Generator().manual_seed(2)).to(DEV) * 100.0
    some = dict(g_logp=g[0], g_entropy=g[1], g_lse=g[2])
    for scale in SCALES:
        print(f"small scales cols={cols} scale={scale} {dtype}", flush=True)
        ref = check(ops.log_probs(x, t, scale=scale, entropy=True, top=top), x, t, top, scale)
        assert scale > 2.0 ** -120 or (ref.p > 0).sum() == torch.isfinite(x).sum()          # nothing is out of reach
        check(ops.log_probs(x, t, scale=scale), x, t, 0, scale)
        norm, h = (torch.from_numpy(v).float().to(DEV) for v in (ref.norm, ref.entropy))
        check_grad(ops.log_probs_grad(x, t, norm, entropy=h, scale=scale, **some), ref, dtype, t, **some)
        check_grad(ops.log_probs_grad(x, t, norm, g_logp=g[0], scale=scale), ref, dtype, t, g_logp=g[0])


def test_two_places_a_small_scale_apart(ops):
    """z = 2 and -2."""
    x = torch.tensor([[2e38, -2e38]], device=DEV, requires_grad=True)
    logp, entropy, lse = target_log_probs(x, torch.tensor([1], device=DEV), ops, scale=1e-38)
    z = x.detach().cpu().double()[0] * float(np.float32(1e-38))
    want = torch.logsumexp(z, 0)
    assert abs(float(lse.detach()) - float(want)) < 1e-6 and abs(float(logp.detach()) - float(z[1] - want)) < 1e-6
    p = torch.softmax(z, 0)
    assert abs(float(entropy.detach()) + float((p * p.log()).sum())) < 1e-6
    (dx,) = torch.autograd.grad(logp.sum(), x)
    # below the normal numbers: steps of 2^-149
    assert ((dx.cpu().double()[0] - 1e-38 * torch.tensor([-float(p[0]), float(p[0])], dtype=torch.float64)).abs() <= 1e-44).all()
