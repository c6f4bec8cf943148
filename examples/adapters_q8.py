"""Adapters of several tasks on one rebuilt network whose weights stay in 8 bits: trained together, and served together.

    python examples/adapters_q8.py

1. a classifier of linear layers goes through one prune-and-compact step and is rebuilt, odd widths and all;
2. its linear tensors are quantised once, a scale per output channel, and stay as they are;
3. low-rank adapters of several tasks are trained beside them: each row of a batch has its task's adapter, the loss is
   the mean log probability of the labels (padded rows are left out), and the adapters' gradients are clipped by
   the norm of all of them;
4. rows of all tasks, and of none, are served in one batch: 8-bit products, adapters from the same 8-bit rows, and of each
   row the likeliest classes with their log probabilities.

Everything runs on one stream; nothing but the prints waits for it."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2309_06973_amd import synth                                      # noqa: E402
from paper_2309_06973_amd.pipeline import Pipeline                          # noqa: E402
from paper_2309_06973_amd.q8 import Q8, adapted, target_log_probs           # noqa: E402


class Classifier:
    """Descriptors of: input, hidden layer, classes.  Groups: 0 input and 1 classes (pinned), 2 hidden channels."""

    def __init__(self, d_in, hidden, classes):
        T, G = synth.TensorDesc, synth.GroupDesc
        self.groups = [G(d_in, 1), G(classes, 1), G(hidden, 0)]
        self.tensors = [T(0, hidden, d_in, 1, 1, 1, 2, 0, 1), T(hidden * d_in, classes, hidden, 1, 1, 1, 1, 2, 1)]
        self.vecs, self.n_vec, self.name = [], 0, "classifier"
        self.n_weights = self.n_prunable = hidden * (d_in + classes)

    def init(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = torch.randn(self.n_weights, generator=g, device="cuda")
        for t in self.tensors:
            scale = torch.exp(torch.randn(t.out_ch, 1, generator=g, device="cuda"))
            w[t.offset:t.offset + t.out_ch * t.in_ch].view(t.out_ch, t.in_ch).mul_(scale * math.sqrt(1.0 / t.in_ch))
        return w, torch.zeros(0, device="cuda")


class Adapted:
    """The rebuilt network in 8 bits with adapters of `tasks` tasks beside each of its layers."""

    def __init__(self, ops, weights, tasks, rank, seed=3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.ops, self.codes = ops, [ops.quantize(w) for w in weights]
        self.values = [ops.dequantize(c, torch.bfloat16) for c in self.codes]          # what the gradient of an input is made with
        make = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
        self.a = [(make(tasks, rank, w.shape[1]) / math.sqrt(w.shape[1])).bfloat16().requires_grad_() for w in weights]
        self.b = [torch.zeros(tasks, w.shape[0], rank, dtype=torch.bfloat16, device="cuda").requires_grad_() for w in weights]
        self.scale = torch.full((tasks,), 2.0, device="cuda")

    def parameters(self):
        return [*self.a, *self.b]

    def train(self, x, task):
        """Logits of bf16 rows, with the adapters' gradients; the weights are constants."""
        for i, w in enumerate(self.values):
            x = adapted(x @ w.t(), x, self.a[i], self.b[i], task, self.ops, scale=self.scale)
            x = torch.relu(x) if i + 1 < len(self.values) else x
        return x

    @torch.no_grad()
    def serve(self, x, task, top):
        """The likeliest classes of bf16 rows: products and adapters read the same 8-bit rows."""
        ops = self.ops
        for i, c in enumerate(self.codes):
            m = ops.quantize(x, relu=i > 0)
            y = ops.matmul(m, c)
            x = ops.adapters(y, m, self.a[i], self.b[i], task, scale=self.scale, out=y)
        return ops.log_probs(x, entropy=True, top=top)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--inputs", type=int, default=256)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--classes", type=int, default=200)
    ap.add_argument("--tasks", type=int, default=4)
    ap.add_argument("--rank", type=int, default=8)
    ap.add_argument("--rows", type=int, default=512)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--sparsity", type=float, default=0.7)
    a = ap.parse_args(argv)
    net, ops = Classifier(a.inputs, a.hidden, a.classes), Q8()

    # 1. pruned and rebuilt
    w, v = net.init(7)
    pl = Pipeline(net, w, v)
    _, (_, tensors, _, (n_w,), _) = pl.step([synth.prune_count(net.n_prunable, a.sparsity)])
    small = [pl.d_w_out[t.offset:t.offset + t.out_ch * t.in_ch].view(t.out_ch, t.in_ch) for t in list(tensors)[:len(net.tensors)]]

    # 2. in 8 bits, with adapters beside
    model = Adapted(ops, small, a.tasks, a.rank)

    # 3. rows of all tasks, each with labels of its own; some positions are padding
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(a.rows, a.inputs, generator=g, device="cuda").bfloat16()
    task = torch.randint(0, a.tasks, (a.rows,), generator=g, device="cuda").sort().values
    label = torch.randint(0, a.classes, (a.rows,), generator=g, device="cuda")
    label[torch.rand(a.rows, generator=g, device="cuda") < 0.1] = -1
    valid, losses, norms = (label >= 0).sum(), [], []
    for _ in range(a.steps):
        logp, _, _ = target_log_probs(model.train(x, task), label, ops)
        loss = -logp.sum() / valid
        grads = list(torch.autograd.grad(loss, model.parameters()))
        norms.append(ops.clip_grad_norm(grads, 1.0))
        with torch.no_grad():
            for p, d in zip(model.parameters(), grads):
                p -= 0.5 * d
        losses.append(loss.detach())

    # 4. all of them served in one batch, and rows without an adapter
    served = torch.where(torch.arange(a.rows, device="cuda") % 16 == 5, -1, task)
    r = model.serve(x, served, min(5, a.classes))
    first, last = (float(losses[0]), float(losses[-1])) if losses else (float("nan"),) * 2
    print(f"{net.n_weights} weights rebuilt to {n_w} in layers of {[tuple(t.shape) for t in small]}, {sum(p.numel() for p in model.parameters())} numbers of adapters")
    print(f"loss {first:.4f} -> {last:.4f} in {a.steps} steps, gradient norm {float(norms[-1]) if norms else float('nan'):.4f} before clipping")
    print(f"likeliest class of the first row: {int(r.index[0, 0])} with log probability {float(r.top[0, 0]):.4f}, entropy {float(r.entropy[0]):.4f}")
    result = dict(first=first, last=last, model=model, served=r, x=x, task=task, label=label, numbers=served, small=small, norms=norms)
    torch.cuda.synchronize()
    pl.close()
    ops.close()
    return result


if __name__ == "__main__":
    main()
