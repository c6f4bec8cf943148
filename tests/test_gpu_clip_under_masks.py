"""A training step under the masks that a prune-and-compact step has written: log probabilities of the labels, the gradients of a
network's tensors where they lie in one arena, and their clipping with the masks as the step left them."""
import math

import pytest
import torch

from paper_2309_06973_amd import synth
from paper_2309_06973_amd.pipeline import Pipeline
from paper_2309_06973_amd.q8 import Q8, target_log_probs
from test_gpu_grad_norm import check

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def pruned():
    spec, w, v = synth.generate_config(1)
    pl = Pipeline(spec, w, v)
    pl.step([synth.prune_count(spec.n_prunable, 0.9)])
    torch.cuda.synchronize()
    yield spec, pl
    torch.cuda.synchronize()
    pl.close()


def test_gradients_of_all_tensors(pruned):
    """Tensors one behind the other, wherever in the arena and in the mask they start."""
    spec, pl = pruned
    arena = torch.randn(spec.w_elems, generator=torch.Generator().manual_seed(1)).to(DEV)
    assert len(spec.tensors) > 2 and all(t.prunable for t in spec.tensors)
    grads = [arena[t.offset:t.offset + t.numel].view(t.out_ch, t.in_ch, t.kh, t.kw) for t in spec.tensors]
    masks = [pl.d_mask[t.offset:t.offset + t.numel].view(t.out_ch, t.in_ch, t.kh, t.kw) for t in spec.tensors]
    assert 0 < sum(int((m != 0).sum()) for m in masks) < spec.n_prunable
    before, mask = [g.clone() for g in grads], pl.d_mask.clone()
    ops = Q8()
    norm = float(ops.grad_norm(grads, masks=masks))
    for max_norm in (0.5 * norm, 2.0 * norm):
        for g, b in zip(grads, before):
            g.copy_(b)
        bound = float(torch.tensor(max_norm, dtype=torch.float32))
        check(ops.clip_grad_norm(grads, max_norm, masks=masks), grads, before, bound, masks)
        assert torch.equal(pl.d_mask, mask)
    torch.cuda.synchronize()
    ops.close()


def test_a_step_that_keeps_what_was_pruned(pruned):
    """The last layer trained on its pruned weights: those stay 0, the others move by the clipped gradient."""
    spec, pl = pruned
    t = spec.tensors[-1]
    rows, cols, here = t.out_ch, t.in_ch, slice(t.offset, t.offset + t.numel)
    sparse, mask = pl.d_w_sparse[here].view(rows, cols), pl.d_mask[here].view(rows, cols)
    weights = sparse.clone().requires_grad_()
    x = torch.randn(100, cols, generator=torch.Generator().manual_seed(2)).to(DEV)
    label = torch.randint(-1, rows, (100,), generator=torch.Generator().manual_seed(3)).to(DEV)
    ops = Q8()
    logp, _, _ = target_log_probs(x @ weights.t(), label, ops)
    (g,) = torch.autograd.grad(-logp.sum(), weights)
    z = (x.cpu().double() @ weights.detach().cpu().double().t()).requires_grad_()
    want = -torch.log_softmax(z, 1)[torch.arange(100), label.cpu().clamp(min=0)][label.cpu() >= 0].sum()
    (dz,) = torch.autograd.grad(want, z)
    full = dz.t() @ x.cpu().double()
    # logits are fp32 sums of 64 products, p is off by their size; sums of 100 products
    off = 2.0 ** -24 * 400 * (dz.abs().t() @ x.cpu().double().abs() + x.cpu().double().abs().sum(0))
    assert ((g.cpu().double() - full).abs() <= off).all()
    kept = g.clone()
    norm = ops.clip_grad_norm([g], 0.25, masks=[mask])
    check(norm, [g], [kept], 0.25, [mask])
    with torch.no_grad():
        weights -= 0.1 * g
    assert (weights.detach()[mask == 0] == 0).all() and (weights.detach()[mask != 0] != sparse[mask != 0]).any()
    assert math.isfinite(float(norm)) and float(norm) > 0.25
    torch.cuda.synchronize()
    ops.close()
