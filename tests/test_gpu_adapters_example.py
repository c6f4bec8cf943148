"""The run of a rebuilt network with adapters: loss, gradients, clipping and serving together."""
import importlib.util
import os

import pytest
import torch

from oracle import learn_oracle as L
from paper_2309_06973_amd.q8 import Q8, target_log_probs

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("adapters_q8", os.path.join(ROOT, "examples", "adapters_q8.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("args", [[], ["--inputs", "100", "--hidden", "333", "--classes", "37", "--tasks", "3", "--rank", "5", "--rows", "77", "--steps", "3"],
                                  ["--tasks", "1", "--rows", "1", "--steps", "2"], ["--steps", "0"]])
def test_runs(example, args):
    r = example.main(args)
    s = r["served"]
    assert all(torch.isfinite(t).all() for t in (s.lse, s.entropy, s.top)) and (s.top[:, 1:] <= s.top[:, :-1]).all()
    assert all(torch.isfinite(n) for n in r["norms"])


def test_gradients(example):
    """The run's gradients against the same network in 64 bits.  The run's activations are bf16, each off by half a step, 2^-8: layers and
    adapters add such errors up, to no more than 2^-4 of a gradient's norm over two layers."""
    r = example.main(["--rows", "200", "--steps", "4", "--hidden", "300", "--classes", "50"])
    model, x, task, label = r["model"], r["x"], r["task"], r["label"]
    ops = Q8()
    model.ops = ops
    logp, _, _ = target_log_probs(model.train(x, task), label, ops)
    valid = (label >= 0).sum()
    got = torch.autograd.grad(-logp.sum() / valid, model.parameters())
    d = lambda t: t.detach().cpu().double()
    a, b = [d(t).requires_grad_() for t in model.a], [d(t).requires_grad_() for t in model.b]
    h, t = d(x), task.cpu()
    for i, w in enumerate(model.values):
        h = h @ d(w).t() + 2.0 * torch.einsum("mr,mnr->mn", torch.einsum("mk,mrk->mr", h, a[i][t]), b[i][t])
        h = torch.relu(h) if i + 1 < len(model.values) else h
    keep = label.cpu() >= 0
    loss = -torch.log_softmax(h, 1)[torch.arange(len(t)), label.cpu().clamp(min=0)][keep].sum() / int(valid)
    for u, v in zip(got, torch.autograd.grad(loss, [*a, *b])):
        assert float((d(u) - v).norm()) <= 2.0 ** -4 * float(v.norm())
    # the same gradients clipped
    norm, want = L.clipped(got, 0.125)
    kept = [u.clone() for u in got]
    assert abs(float(ops.clip_grad_norm(kept, 0.125)) - norm) <= 1.01 * L.U * norm
    for u, w in zip(kept, want):
        assert ((u.cpu().double() - w).abs() <= (L.HALF_STEP[u.dtype] + 2 * L.U) * w.abs() + L.LEAST[u.dtype]).all()
    torch.cuda.synchronize()
    ops.close()
