"""What the 8-bit operators' calls owe to autograd: a tensor that they write has a new version."""
import pytest
import torch

from paper_2309_06973_amd import q8


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
