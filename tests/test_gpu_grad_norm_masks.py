"""Gradients and masks in one arena: what is written may not lie over a mask, whichever tensor it belongs to."""
import pytest
import torch

from paper_2309_06973_amd import shifter as S
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


def test_what_is_written_over_a_mask_is_refused(ops):
    arena = torch.ones(4096, dtype=torch.uint8, device=DEV)
    values = lambda a, n: arena[a:a + 4 * n].view(torch.float32)
    other = torch.ones(100, device=DEV)
    for grads, masks, out in (([values(0, 100)], [arena[399:499]], None), ([values(400, 100)], [arena[301:401]], None), ([values(400, 100)], [arena[500:600]], None),
                              ([other], [arena[0:100]], [values(96, 100)]), ([values(0, 100), other], [None, arena[200:300]], None),
                              ([other, values(1000, 100)], [arena[1300:1400], None], [torch.ones(100, device=DEV), values(1000, 100)])):
        before = arena.clone()
        with pytest.raises(S.ShifterError, match="overlaps"):
            ops.clip_grad_norm(grads, 1.0, masks=masks, out=out)
        assert torch.equal(arena, before) and (other == 1).all()


def test_masks_beside_what_is_written(ops):
    """One mask for two tensors, masks that begin where a tensor ends, and one over elements that are only read."""
    arena = torch.zeros(4096, dtype=torch.uint8, device=DEV)
    values = lambda a, n: arena[a:a + 4 * n].view(torch.float32)
    a, b = values(0, 100), values(600, 50)
    arena[400:600] = (torch.arange(200, device=DEV) % 3 > 0).to(torch.uint8)
    a.copy_(torch.linspace(-3, 3, 100, device=DEV))
    b.copy_(torch.linspace(1, 2, 50, device=DEV))
    before = [a.clone(), b.clone()]
    masks = [arena[400:500], arena[450:500]]
    kept = arena[400:600].clone()
    check(ops.clip_grad_norm([a, b], 0.5, masks=masks), [a, b], before, 0.5, masks)
    assert torch.equal(arena[400:600], kept)
    out = [torch.empty(100, device=DEV)]
    check(ops.clip_grad_norm([a], 0.1, masks=[arena[0:100]], out=out), out, [a], 0.1, [arena[0:100]])
    check(ops.grad_norm([a], masks=[arena[0:100]]), None, [a], 1.0, [arena[0:100]])
