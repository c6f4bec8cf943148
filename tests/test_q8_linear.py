"""checkpointed_linear without a GPU: its autograd function over the operators' definition on the CPU."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as Q
from paper_2309_06973_amd import shifter as S
from paper_2309_06973_amd.q8 import Q8Matrix, checkpointed_linear


class Definition:
    """quantize and weight_grad of Q8, from the definition in 64 bits."""

    def quantize(self, x):
        assert x.dim() == 2 and (x.shape[1] < 2 or x.stride(1) == 1) and (x.shape[0] < 2 or x.stride(0) >= x.shape[1])
        q, s = Q.quantize(x)
        codes = torch.zeros((q.shape[0], -(-q.shape[1] // 16) * 16), dtype=torch.int8)
        codes[:, :q.shape[1]] = torch.from_numpy(q)
        return Q8Matrix(codes, torch.from_numpy(np.atleast_1d(s).astype(np.float32)), q.shape[1])

    def weight_grad(self, g, x, mask=None, out=None, accumulate=False):
        assert g.shape[0] == x.rows <= S.SHIFTER_Q8_MAX_SUM
        assert mask is None or (mask.dtype == torch.uint8 and mask.stride(1) == 1 and mask.stride(0) >= mask.shape[1])
        d, _ = Q.weight_grad(g, x.q[:, :x.cols].numpy(), x.scale.numpy(), None if mask is None else mask.numpy())
        d = torch.from_numpy(d).float()
        if out is None:
            return d
        return out.copy_(torch.where(mask == 0, out, out + d) if accumulate and mask is not None else out + d if accumulate else d)


OPS = Definition()


def operands(m, n, k, seed=0, **kw):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(*s, generator=g).to(**kw).requires_grad_() for s in ((m, k), (n, k))]


def gradients(x, w, layer, loss):
    return torch.autograd.grad(loss(layer(x, w)), (x, w), create_graph=True)


def ours(x, w):
    return checkpointed_linear(x, w, OPS)


LOSSES = {"square": lambda y: y.square().sum(), "linear": lambda y: y.sum()}


@pytest.mark.parametrize("loss", LOSSES)
@pytest.mark.parametrize("beside", [False, True])
def test_second_derivatives_of_the_weights_gradient_are_refused(loss, beside):
    """A penalty on the gradients: those of the weights have no derivative of their own, which is an error and not a
    term left out in silence, also where the penalty reaches the operands on other ways."""
    x, w = operands(6, 5, 4)
    dx, dw = gradients(x, w, ours, LOSSES[loss])
    penalty = dx.square().sum() + dw.square().sum() + (LOSSES[loss](x @ w.t()) if beside else 0.0)
    for inputs in ((x,), (w,), (x, w)):
        with pytest.raises(RuntimeError, match="no derivative of its own"):
            torch.autograd.grad(penalty, inputs, retain_graph=True, allow_unused=True)
    with pytest.raises(RuntimeError, match="no derivative of its own"):
        penalty.backward()


@pytest.mark.parametrize("loss", LOSSES)
def test_second_derivatives_of_the_inputs_gradient(loss):
    """They are torch's, but for what goes on to the weights, from the 8-bit input: half a code of each row off at most.
    First derivatives do not mind the graph."""
    x, w = operands(6, 5, 4)
    dx, dw = gradients(x, w, ours, LOSSES[loss])
    plain = gradients(x, w, lambda x, w: x @ w.t(), LOSSES[loss])
    got, want = (torch.autograd.grad(d.square().sum(), (x, w), allow_unused=True) for d in (dx, plain[0]))
    for a, b in zip(got[:1], want[:1]):
        assert (a is None or not a.any()) if b is None else torch.equal(a, b)
    scale = OPS.quantize(x.detach()).scale[:, None]
    # the way through y in the square's case: y's gradient is 2 y, dx is 2 y w, the penalty's with respect to y 4 dx w'
    off = ((4.0 * dx.detach() @ w.detach().t()).abs().t() @ (0.5 * scale).expand(6, 4)) if loss == "square" else 0.0
    assert ((got[1] - want[1]).abs() <= off + 32 * Q.U32 * want[1].abs().max()).all()
    for a, b in zip((dx, dw), torch.autograd.grad(LOSSES[loss](ours(x, w)), (x, w))):
        assert torch.equal(a, b)
    assert torch.equal(dx, plain[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("inside", [False, True])
def test_autocast(dtype, inside):
    """The product in bf16 as torch's own; gradients in the operands' types, whether the backward pass runs in the region or not."""
    x, w = operands(6, 5, 4)
    x = x.detach().to(dtype).requires_grad_()
    grads = []
    for layer in (ours, lambda x, w: x @ w.t()):
        x.grad = w.grad = None
        with torch.autocast("cpu", dtype=torch.bfloat16):
            y = layer(x, w)
            loss = y.float().square().sum()
            if inside:
                loss.backward()
        if not inside:
            loss.backward()
        grads.append((y.detach(), x.grad, w.grad))
    (y, dx, dw), (y2, dx2, _) = grads
    assert y.dtype == torch.bfloat16 and torch.equal(y, y2)
    assert dx.dtype == dtype and torch.equal(dx, dx2)
    m = OPS.quantize(x.detach())
    assert dw.dtype == torch.float32 and torch.equal(dw, OPS.weight_grad((2.0 * y.float()).bfloat16(), m))


@pytest.mark.parametrize("rows", [7, 8, 9, 16, 17, 30])
@pytest.mark.parametrize("masked", [False, True])
def test_more_rows_than_one_sum_holds(monkeypatch, rows, masked):
    """The weights' gradient of more rows than a call takes is that of several, added up: an fp32 rounding a part more."""
    x, w = operands(rows, 5, 4)
    mask = (torch.arange(20).view(5, 4) % 3 > 0).to(torch.uint8) if masked else None
    y = checkpointed_linear(x, w, OPS, mask)
    g = torch.randn(y.shape, generator=torch.Generator().manual_seed(1))
    monkeypatch.setattr(S, "SHIFTER_Q8_MAX_SUM", 8)
    dx, dw = torch.autograd.grad(y, (x, w), g)
    q, s = Q.quantize(x)
    want, _ = Q.weight_grad(g, q, s.astype(np.float32), None if mask is None else mask.numpy())
    size, _ = Q.weight_grad(g.abs(), np.abs(q), s.astype(np.float32))
    parts = -(-rows // 8)
    assert (np.abs(Q.f64(dw) - want) <= 2 * parts * Q.U32 * size).all()
    assert torch.equal(dx, g @ w.detach())


def layouts(x):
    """The values of x [24, 4] in shapes and orders that a layer meets."""
    yield "columns apart", x.t().contiguous().t()
    yield "every other column", torch.stack([x, -x], 2).view(24, 8)[:, ::2]
    yield "one row for all", x[:1].expand(24, 4)
    yield "batch of sequences", x.view(2, 3, 4, 4)
    yield "sequences first", x.view(4, 6, 4).transpose(0, 1)
    yield "one token", x[3]
    yield "one token, columns apart", torch.stack([x, x], 2)[5, :, 0]
    yield "no tokens", x[:0].view(3, 0, 4)


@pytest.mark.parametrize("which", range(8))
def test_layouts_of_the_input(which):
    base, w = operands(24, 5, 4)
    name, x = list(layouts(base.detach()))[which]
    x = x.requires_grad_()
    y = checkpointed_linear(x, w, OPS)
    # four or five terms, a rounding each and one for each sum, in whatever order the products take
    near = lambda got, a, b: (got.detach().double() - a.double() @ b.double()).abs() <= 5 * Q.U32 * (a.abs().double() @ b.abs().double())
    assert near(y, x.detach(), w.detach().t()).all(), name
    g = torch.randn(y.shape, generator=torch.Generator().manual_seed(2))
    dx, dw = torch.autograd.grad(y, (x, w), g)
    assert dx.shape == x.shape and near(dx, g, w.detach()).all()
    rows = x.detach().reshape(-1, 4).contiguous()
    assert torch.equal(dw, OPS.weight_grad(g.reshape(-1, 5), OPS.quantize(rows)))


def test_masks():
    """One that the backward pass could not use is refused where it is given; the order of its memory does not matter."""
    x, w = operands(6, 5, 4)
    mask = (torch.arange(20).view(5, 4) % 3 > 0).to(torch.uint8)
    for bad in (mask.bool(), mask.float(), mask[:4], mask[:, :3], mask.t(), mask.to("meta")):
        with pytest.raises(ValueError, match="mask"):
            checkpointed_linear(x, w, OPS, bad)
    want = torch.autograd.grad(checkpointed_linear(x, w, OPS, mask).sum(), (w,))[0]
    for same in (mask.t().contiguous().t(), torch.stack([mask, 1 - mask], 2)[:, :, 0]):
        assert torch.equal(torch.autograd.grad(checkpointed_linear(x, w, OPS, same).sum(), (w,))[0], want)
    row = torch.ones(1, 4, dtype=torch.uint8).expand(5, 4)
    assert torch.equal(torch.autograd.grad(checkpointed_linear(x, w, OPS, row).sum(), (w,))[0],
                       torch.autograd.grad(checkpointed_linear(x, w, OPS).sum(), (w,))[0])
