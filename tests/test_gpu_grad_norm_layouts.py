"""Masks and results that lie in memory as their gradient does, whatever strides their dimensions of one element have."""
import pytest
import torch

from oracle import learn_oracle as L
from paper_2309_06973_amd.q8 import Q8
from test_gpu_grad_norm import check

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ops():
    o = Q8()
    yield o
    torch.cuda.synchronize()
    o.close()


def alike(shape, strides, dtype, seed):
    """A tensor of these strides over as many elements as it has, in an arena of their own."""
    n = torch.Size(shape).numel()
    v = torch.randn(n, generator=torch.Generator().manual_seed(seed)).to(DEV)
    v = (v > 0).to(dtype) if dtype == torch.uint8 else v.to(dtype)
    return torch.as_strided(v, shape, strides)


@pytest.mark.parametrize("shape, one, other", [((16, 8, 1, 1), (8, 1, 8, 8), (8, 1, 1, 1)), ((1, 700), (700, 1), (1, 1)), ((300, 1), (1, 1), (1, 300)),
                                               ((1, 1, 1), (1, 1, 1), (9, 7, 5)), ((3, 1, 50), (50, 999, 1), (50, 50, 1)), ((1, 5, 7), (35, 1, 5), (2, 1, 5))])
def test_dimensions_of_one_element(ops, shape, one, other):
    for dtype in (torch.float32, torch.bfloat16):
        g, m, out = alike(shape, one, dtype, 1), alike(shape, other, torch.uint8, 2), alike(shape, other, dtype, 3)
        for masks in (None, [m]):
            check(ops.grad_norm([g], masks=masks), None, [g], 1.0, masks)
            n = ops.clip_grad_norm([g], 0.5, masks=masks, out=[out])
            check(n, [out], [g], 0.5, masks)
        same = g.clone(memory_format=torch.preserve_format)
        ops.clip_grad_norm([same], 0.5, masks=[m])
        assert torch.equal(same, out)


def test_a_pruned_convolution_of_single_places(ops):
    """A channels-last network's 1 x 1 kernels, with masks as they are written: one behind the other."""
    w = torch.randn(16, 8, 1, 1, device=DEV).to(memory_format=torch.channels_last).requires_grad_()
    x = torch.randn(2, 8, 5, 5, device=DEV).to(memory_format=torch.channels_last)
    torch.nn.functional.conv2d(x, w).square().sum().backward()
    mask = (torch.rand(16, 8, 1, 1, device=DEV) < 0.5).to(torch.uint8)
    g = torch.as_strided(w.grad.clone(), (16, 8, 1, 1), (8, 1, 8, 8))
    want, (clipped,) = L.clipped([g], 1.0, [mask])
    assert abs(float(ops.clip_grad_norm([g], 1.0, masks=[mask])) - want) <= 1e-6 * want
    assert ((g.cpu().double() - clipped).abs() <= 1e-6 * clipped.abs()).all()


@pytest.mark.parametrize("shape, one, other", [((4, 6), (6, 1), (1, 4)), ((2, 3, 4), (12, 4, 1), (12, 1, 3)), ((4, 1, 6), (6, 6, 1), (1, 4, 4))])
def test_another_order_is_refused(ops, shape, one, other):
    g = alike(shape, one, torch.float32, 1)
    with pytest.raises(ValueError, match="mask 0"):
        ops.grad_norm([g], masks=[alike(shape, other, torch.uint8, 2)])
    with pytest.raises(ValueError, match="out 0"):
        ops.clip_grad_norm([g], 1.0, out=[alike(shape, other, torch.float32, 3)])
    with pytest.raises(ValueError, match="mask 0"):
        ops.grad_norm([g], masks=[alike(shape, one, torch.uint8, 2).reshape(-1)])
