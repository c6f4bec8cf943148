"""What the 8-bit operators' calls owe to autograd: a tensor that they write has a new version, and a gradient that
they would lose is an error, of the backward pass, or of the call where it writes a given tensor.  The latter needs no GPU:
host tensors are refused for that only afterwards."""
import os

import pytest
import torch

from paper_2309_06973_amd import q8, shifter as S

F32 = torch.float32


@pytest.fixture(scope="module")
def calls():
    if not (os.path.exists(q8._CALLS_PATH) and os.path.exists(S._LIB_PATH)):
        from paper_2309_06973_amd import build
        build.build_library(verbose=False)
    return q8.load_calls()


def codes(rows, cols):
    return q8.Q8Matrix(torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.int8), torch.zeros(rows), cols)


def grad(*shape):
    return torch.ones(*shape, requires_grad=True)


X, W = torch.zeros(3, 4), torch.zeros(4)
LOST = {"rms_norm of x": lambda c: c.rms_norm(0, 0, grad(3, 4), W, 1e-6, X, X, None),
        "rms_norm of residual": lambda c: c.rms_norm(0, 0, X, W, 1e-6, grad(3, 4), X, None),
        "rms_norm to h": lambda c: c.rms_norm(0, 0, X, W, 1e-6, X, grad(3, 4), None),
        "matmul's bias": lambda c: c.matmul(0, 0, codes(3, 5), codes(4, 5), grad(4), False, F32, torch.zeros(3, 4)),
        "weight_grad of g": lambda c: c.weight_grad(0, 0, grad(3, 4), codes(3, 5), None, F32, torch.zeros(4, 5), False, None)}


@pytest.mark.parametrize("which", LOST)
def test_gradients_that_would_be_lost(calls, which):
    with pytest.raises(ValueError, match="needs a gradient"):
        LOST[which](calls)
    with torch.no_grad(), pytest.raises(ValueError, match="is not on cuda:0"):     # the next check
        LOST[which](calls)


def test_what_keeps_its_graph_or_has_none(calls):
    """An 8-bit matrix is a constant, without a residual the stream is x itself, and a new tensor has an error in its graph."""
    for call in (lambda: calls.quantize(0, 0, grad(3, 4), False, None),
                 lambda: calls.rms_norm(0, 0, grad(3, 4), grad(4), 1e-6, None, None, None),
                 lambda: calls.rms_norm(0, 0, grad(3, 4), W, 1e-6, X, None, None),
                 lambda: calls.weight_grad(0, 0, grad(3, 4), codes(3, 5), None, F32, None, False, None)):
        with pytest.raises(ValueError, match="is not on cuda:0"):
            call()


@pytest.fixture(scope="module")
def ops():
    o = q8.Q8()
    yield o
    torch.cuda.synchronize()
    o.close()


@pytest.mark.gpu
def test_versions(ops):
    dev = "cuda"
    x, r, w = torch.randn(5, 40, device=dev), torch.randn(5, 40, device=dev), torch.ones(40, device=dev)
    m, d, dw = ops.quantize(x), torch.empty(5, 40, device=dev), torch.empty(40, 40, device=dev)
    c = torch.empty(5, 5, device=dev)
    for call, outs in ((lambda: ops.quantize(x, out=m), (m.q, m.scale)), (lambda: ops.dequantize(m, out=d), (d,)),
                       (lambda: ops.rms_norm(x, w, 1e-6, residual=r, h=x, out=m), (x, m.q, m.scale)),
                       (lambda: ops.matmul(m, m, out=c), (c,)), (lambda: ops.weight_grad(x, m, out=dw), (dw,)),
                       (lambda: ops.weight_grad(x, m, out=dw, accumulate=True), (dw,))):
        others = [t for t in (x, r, w, m.q, m.scale, d, dw, c) if not any(t is o for o in outs)]
        before = [[t._version for t in ts] for ts in (outs, others)]
        call()
        assert all(t._version > v for t, v in zip(outs, before[0]))
        assert [t._version for t in others] == before[1]
    with torch.inference_mode():
        held = torch.empty(5, 40, device=dev)
        assert torch.equal(ops.dequantize(m, out=held), ops.dequantize(m))
    assert torch.equal(ops.dequantize(m, out=held), ops.dequantize(m))          # no version to be raised


@pytest.mark.gpu
def test_a_saved_tensor_that_is_written(ops):
    x = torch.randn(5, 40, device="cuda")
    w = torch.ones(40, device="cuda", requires_grad=True)
    y = (x * w).sum()                          # keeps x
    ops.rms_norm(x, torch.ones(40, device="cuda"), 1e-6, residual=torch.randn_like(x), h=x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


@pytest.mark.gpu
def test_the_backward_pass_of_a_new_tensor(ops):
    """Such calls run as they are, and say in a backward pass, on every way, that they have no gradient."""
    dev = "cuda"
    x, r, bias = (torch.randn(*s, device=dev) for s in ((5, 40), (5, 40), (7,)))
    w, weights = torch.ones(40, device=dev), ops.quantize(torch.randn(7, 40, device=dev))
    g, m = torch.randn(5, 7, device=dev), ops.quantize(x)
    for call, inputs in ((lambda x, r: ops.rms_norm(x, w, 1e-6, residual=r)[1], (x, r)),
                         (lambda r, x: ops.rms_norm(x, w, 1e-6, residual=r)[1], (r, x)),
                         (lambda b: ops.matmul(m, weights, bias=b, dtype=torch.float32), (bias,)),
                         (lambda g: ops.weight_grad(g, m), (g,))):
        want = call(*inputs)
        assert not want.requires_grad
        leaf = inputs[0].clone().requires_grad_()
        for first in (leaf, leaf * 1.0):       # a leaf, and what is made from it
            got = call(first, *inputs[1:])
            assert torch.equal(got, want) and got.requires_grad
            for loss in (got.square().sum(), got.sum() + leaf.sum()):
                with pytest.raises(RuntimeError, match="passes no gradients on"):
                    torch.autograd.grad(loss, leaf, retain_graph=True)
        with torch.no_grad():
            assert not call(leaf, *inputs[1:]).requires_grad
    assert not ops.quantize(x.clone().requires_grad_()).scale.requires_grad
    leaf = x.clone().requires_grad_()
    assert ops.rms_norm(leaf, w, 1e-6)[1] is leaf
