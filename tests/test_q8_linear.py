"""checkpointed_linear without a GPU: its autograd function over the operators' definition on the CPU."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as Q
from paper_2309_06973_amd.q8 import Q8Matrix, checkpointed_linear


class Definition:
    """quantize and weight_grad of Q8, from the definition in 64 bits."""

    def quantize(self, x):
        q, s = Q.quantize(x)
        codes = np.zeros((q.shape[0], -(-q.shape[1] // 16) * 16), dtype=np.int8)
        codes[:, :q.shape[1]] = q
        return Q8Matrix(torch.from_numpy(codes), torch.from_numpy(np.atleast_1d(s).astype(np.float32)), q.shape[1])

    def weight_grad(self, g, x, mask=None):
        d, _ = Q.weight_grad(g, x.q[:, :x.cols].numpy(), x.scale.numpy(), None if mask is None else mask.numpy())
        return torch.from_numpy(d).float()


OPS = Definition()


def operands(m, n, k, seed=0, **kw):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(*s, generator=g).to(**kw).requires_grad_() for s in ((m, k), (n, k))]


def test_second_derivatives_are_refused():
    """A penalty on the gradients: those of the weights have no derivative of their own, which is an error and not a
    term left out in silence."""
    x, w = operands(6, 5, 4)
    dx, dw = torch.autograd.grad(checkpointed_linear(x, w, OPS).square().sum(), (x, w), create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        torch.autograd.grad(dx.square().sum() + dw.square().sum(), (x, w))
    # first derivatives do not mind the graph
    x2, w2 = (t.detach().requires_grad_() for t in (x, w))
    for a, b in zip((dx, dw), torch.autograd.grad(checkpointed_linear(x2, w2, OPS).square().sum(), (x2, w2))):
        assert torch.equal(a, b)
