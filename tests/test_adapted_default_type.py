"""adapted without a GPU: what it hands to the handle's call is of the types that the call takes, whatever type torch makes
by default."""
import pytest
import torch

from paper_2309_06973_amd import q8


class Handle:
    """Stands in for Q8: keeps what it is given."""

    def adapters(self, y, x, a, b, which, scale=None, out=None, down=None):
        self.down = down
        return y + 1

    def adapters_grad(self, g, x, a, b, which, scale=None, down=None, dx=True):
        assert down is self.down or torch.equal(down, self.down)
        return torch.zeros_like(x) if dx else None, torch.zeros(a.shape, dtype=torch.float32), torch.zeros(b.shape, dtype=torch.float32)


@pytest.mark.parametrize("default", [torch.float32, torch.float64, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_what_is_kept_for_the_gradient_is_fp32(monkeypatch, dtype, default):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    y, x = torch.zeros(3, 5, dtype=dtype), torch.zeros(3, 7, dtype=dtype)
    a, b = torch.zeros(2, 4, 7, dtype=dtype, requires_grad=True), torch.zeros(2, 5, 4, dtype=dtype)
    handle, was = Handle(), torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        out = q8.adapted(y, x, a, b, torch.zeros(3, dtype=torch.int64), handle)
        out.float().sum().backward()
    finally:
        torch.set_default_dtype(was)
    assert handle.down.dtype == torch.float32 and handle.down.shape == (3, 4) and a.grad.dtype == dtype
