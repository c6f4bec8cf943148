"""checkpointed_linear on the device: autocast, more rows than a sum holds, second derivatives.
The weights' gradient is compared with the bound that the interface states, worked out per entry."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as Q
from paper_2309_06973_amd import shifter as S
from paper_2309_06973_amd.q8 import Q8, checkpointed_linear

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ops():
    o = Q8()
    yield o
    torch.cuda.synchronize()
    o.close()


def operands(m, n, k, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [torch.randn(*s, generator=g, device=DEV).requires_grad_() for s in ((m, k), (n, k))]


def near(dw, g, x, mask=None, more=0.0):
    """dw within the stated bound of its definition, `more` half steps of fp32 of the terms' magnitude beside it."""
    q, s = Q.quantize(x)
    s = s.astype(np.float32)
    want, bound = Q.weight_grad(g, q, s, mask)
    size, _ = Q.weight_grad(g.abs(), np.abs(q), s)
    return (np.abs(Q.f64(dw) - want) <= 1.001 * bound + more * Q.U32 * size).all()


@pytest.mark.parametrize("inside", [False, True])
def test_autocast(ops, inside):
    x, w = operands(300, 70, 45)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        y = checkpointed_linear(x, w, ops)
        loss = y.float().square().sum()
        if inside:
            loss.backward()
    if not inside:
        loss.backward()
    g = (2.0 * y.detach().float()).bfloat16()
    assert y.dtype == torch.bfloat16 and torch.equal(x.grad, (g @ w.detach().bfloat16()).float())
    assert w.grad.dtype == torch.float32 and near(w.grad, g, x)


def test_more_rows_than_one_sum_holds(ops):
    rows = S.SHIFTER_Q8_MAX_SUM + 300
    x, w = operands(rows, 33, 40)
    mask = (torch.rand(33, 40, device=DEV) < 0.5).to(torch.uint8)
    y = checkpointed_linear(x, w, ops, mask)
    g = torch.randn_like(y)
    y.backward(g)
    assert near(w.grad, g, x, mask.cpu().numpy(), more=2.0)


def test_second_derivatives(ops):
    x, w = operands(60, 50, 40)
    dx, dw = torch.autograd.grad(checkpointed_linear(x, w, ops).square().sum(), (x, w), create_graph=True)
    with pytest.raises(RuntimeError, match="no derivative of its own"):
        torch.autograd.grad(dx.square().sum() + dw.square().sum() + (x @ w.t()).sum(), (x, w), retain_graph=True)
    # that of the inputs' gradient 2 x w' w is torch's, up to the order of fp32 sums
    got, = torch.autograd.grad(dx.square().sum(), (x,))
    x64, w64 = x.detach().double(), w.detach().double()
    want = 8.0 * x64 @ w64.t() @ w64 @ w64.t() @ w64
    size = 8.0 * x64.abs() @ w64.abs().t() @ w64.abs() @ w64.abs().t() @ w64.abs()
    # four products of sums of 40 to 50 terms, a half step a term and product
    assert ((got.double() - want).abs() <= 4 * 52 * Q.U32 * size).all()


def test_layouts_of_the_input(ops):
    x, w = operands(90, 50, 41)
    g = torch.randn(90, 50, device=DEV)
    for y_of, rows in ((lambda t: t.t().contiguous().t(), x), (lambda t: t.view(6, 15, 41), x),
                       (lambda t: t.view(9, 10, 41).transpose(0, 1), x.view(9, 10, 41).transpose(0, 1).reshape(90, 41))):
        y = checkpointed_linear(y_of(x), w, ops)
        dx, dw = torch.autograd.grad(y, (x, w), g.view(y.shape))
        assert y.shape == y_of(x).shape[:-1] + (50,) and dx.shape == x.shape
        assert near(dw, g, rows)
