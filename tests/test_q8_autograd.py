"""What the 8-bit operators' calls owe to autograd: a tensor that they write has a new version, and a gradient that
they would lose is refused.  The refusals need no GPU: host tensors are refused for that only afterwards."""
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
LOST = {"rms_norm of x": lambda c: c.rms_norm(0, 0, grad(3, 4), W, 1e-6, X, None, None),
        "rms_norm of residual": lambda c: c.rms_norm(0, 0, X, W, 1e-6, grad(3, 4), None, None),
        "rms_norm to h": lambda c: c.rms_norm(0, 0, X, W, 1e-6, X, grad(3, 4), None),
        "matmul's bias": lambda c: c.matmul(0, 0, codes(3, 5), codes(4, 5), grad(4), False, F32, None),
        "weight_grad of g": lambda c: c.weight_grad(0, 0, grad(3, 4), codes(3, 5), None, F32, None, False, None)}


@pytest.mark.parametrize("which", LOST)
def test_gradients_that_would_be_lost(calls, which):
    with pytest.raises(ValueError, match="needs a gradient"):
        LOST[which](calls)
    with torch.no_grad(), pytest.raises(ValueError, match="is not on cuda:0"):     # the next check
        LOST[which](calls)


def test_what_keeps_its_graph_or_has_none(calls):
    """An 8-bit matrix is a constant, and without a residual the stream is x itself."""
    for call in (lambda: calls.quantize(0, 0, grad(3, 4), False, None),
                 lambda: calls.rms_norm(0, 0, grad(3, 4), grad(4), 1e-6, None, None, None)):
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
