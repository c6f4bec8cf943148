"""A residual network of linear layers, pruned, trained on under its mask, rebuilt and served in 8 bits.

    python examples/residual_mlp_q8.py

1. one prune-and-compact step gives the sparse weights, the mask and the plan;
2. the sparse network trains on: every linear layer keeps its input as an 8-bit checkpoint, and its
   weight gradient, read from that, is zero where a weight was pruned (Sec. III-C: weights stay
   masked between two prunings);
3. the trained network goes through the step again and is rebuilt without its dead channels;
4. the rebuilt linear tensors, odd widths and all, are quantised a scale per output channel, and
   tokens are served through RMS norm, 8-bit product, ReLU, 8-bit product, residual.

Everything runs on one stream; nothing but the prints waits for it."""
import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2309_06973_amd import synth                                      # noqa: E402
from paper_2309_06973_amd.pipeline import Pipeline                          # noqa: E402
from paper_2309_06973_amd.q8 import Q8, checkpointed_linear                 # noqa: E402

EPS = 1e-6


class Net:
    """Descriptors of: input -> stream; blocks of norm, up, ReLU, down added to the stream; norm, output.
    Groups: 0 input and 1 output (pinned), 2 the stream, 3.. each block's hidden channels."""

    def __init__(self, d_in=64, stream=512, hidden=1024, blocks=3, d_out=96):
        T, V, G = synth.TensorDesc, synth.VecDesc, synth.GroupDesc
        self.groups = [G(d_in, 1), G(d_out, 1), G(stream, 0)] + [G(hidden, 0) for _ in range(blocks)]
        self.tensors, self.vecs = [], []
        layers = [(2, 0)] + [p for b in range(blocks) for p in ((3 + b, 2), (2, 3 + b))] + [(1, 2)]
        offset = 0
        for out, inp in layers:
            o, i = self.groups[out].width, self.groups[inp].width
            self.tensors.append(T(offset, o, i, 1, 1, 1, out, inp, 1))
            offset += o * i
        self.n_weights = self.n_prunable = offset
        offset = 0
        for group in [2] * (blocks + 1) + [3 + b for b in range(blocks)]:   # norm weights, then the up layers' biases
            self.vecs.append(V(offset, self.groups[group].width, group))
            offset += self.groups[group].width
        self.n_vec, self.blocks, self.name = offset, blocks, "residual_mlp"

    def init(self, seed):
        """Kaiming-normal weights times a heavy-tailed scale per output channel, so that channels die."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = torch.randn(self.n_weights, generator=g, device="cuda")
        for t in self.tensors:
            scale = torch.exp(torch.randn(t.out_ch, 1, generator=g, device="cuda"))
            w[t.offset:t.offset + t.out_ch * t.in_ch].view(t.out_ch, t.in_ch).mul_(scale * math.sqrt(1.0 / t.in_ch))
        v = torch.ones(self.n_vec, device="cuda")
        v[(self.blocks + 1) * self.groups[2].width:] = 0.0
        return w, v


def split(tensors, vecs, w, v):
    """([weight matrix], [vector]) of arenas with these descriptors."""
    n = lambda d: getattr(d, "length", getattr(d, "len", 0))
    return ([w[t.offset:t.offset + t.out_ch * t.in_ch].view(t.out_ch, t.in_ch) for t in tensors],
            [v[d.offset:d.offset + n(d)] for d in vecs])


def forward(x, w, v, blocks, linear):
    """The network in floating point."""
    def norm(h, weight):
        return h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * weight
    h = linear(x, w[0], 0)
    for b in range(blocks):
        u = torch.relu(linear(norm(h, v[b]), w[1 + 2 * b], 1 + 2 * b) + v[blocks + 1 + b])
        h = h + linear(u, w[2 + 2 * b], 2 + 2 * b)
    return linear(norm(h, v[blocks]), w[-1], len(w) - 1)


class Served:
    """A rebuilt variant with its linear tensors in 8 bits."""

    def __init__(self, ops, net, w, v):
        self.ops, self.blocks = ops, net.blocks
        self.w = [ops.quantize(t) for t in w]
        # the norm's mean counted the stream's dead channels, which are zero: fewer channels, larger mean
        share = net.groups[2].width / max(1, w[0].shape[0])
        self.eps = EPS * share
        self.norms = [t * math.sqrt(share) for t in v[:net.blocks + 1]]
        self.biases = [t.contiguous() for t in v[net.blocks + 1:]]

    def __call__(self, x):
        """x: bf16 tokens.  A block's output and the stream meet in the next norm's addition."""
        ops = self.ops
        h = ops.matmul(ops.quantize(x), self.w[0])
        added = None
        for b in range(self.blocks):
            m, h = ops.rms_norm(h, self.norms[b], self.eps, residual=added, h=h if added is not None else None)
            u = ops.quantize(ops.matmul(m, self.w[1 + 2 * b], bias=self.biases[b]), relu=True)
            added = ops.matmul(u, self.w[2 + 2 * b])
        m, _ = ops.rms_norm(h, self.norms[-1], self.eps, residual=added, h=h if added is not None else None)
        return ops.matmul(m, self.w[-1], dtype=torch.float32)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--stream", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--blocks", type=int, default=3)
    ap.add_argument("--sparsity", type=float, default=0.8)
    ap.add_argument("--steps", type=int, default=20, help="training steps between the two prunings")
    ap.add_argument("--tokens", type=int, default=256)
    a = ap.parse_args(argv)
    torch.manual_seed(1)
    net = Net(stream=a.stream, hidden=a.hidden, blocks=a.blocks)
    w, v = net.init(7)
    n_prune = synth.prune_count(net.n_prunable, a.sparsity)
    ops = Q8()

    # 1. mask and sparse weights
    pl = Pipeline(net, w, v)
    pl.step([n_prune])
    masks = [m.view(t.out_ch, t.in_ch) for t, m in zip(net.tensors, pl.d_mask[:net.n_weights].split(
        [t.out_ch * t.in_ch for t in net.tensors]))]

    # 2. training on under the mask, inputs kept in 8 bits
    arena = pl.d_w_sparse.clone()
    weights, vectors = split(net.tensors, net.vecs, arena, v)
    for t in weights:
        t.requires_grad_()
    x = torch.randn(a.tokens, net.groups[0].width, device="cuda")
    target = torch.randn(a.tokens, net.groups[1].width, device="cuda")
    losses = []
    for _ in range(a.steps):
        y = forward(x, weights, vectors, net.blocks, lambda h, t, i: checkpointed_linear(h, t, ops, masks[i]))
        loss = (y - target).square().mean()
        for t, g in zip(weights, torch.autograd.grad(loss, weights)):
            with torch.no_grad():
                t -= 0.05 * g / (g.norm() + 1e-12)
        losses.append(loss.detach())
    arena = arena.detach()

    # 3. the trained weights through the step again, rebuilt
    pl2 = Pipeline(net, arena, v)
    _, (_, tensors, vecs, (n_w,), (n_v,)) = pl2.step([n_prune])
    dead = [g.width - int(n) for g, n in zip(net.groups, pl2.d_new_width.cpu())]
    small = split(list(tensors)[:len(net.tensors)], list(vecs)[:len(net.vecs)], pl2.d_w_out[:n_w], pl2.d_vecs_out[:n_v])

    # 4. served in 8 bits
    served = Served(ops, net, *small)
    tokens = x.bfloat16()
    got = served(tokens)
    with torch.no_grad():
        full, vec = split(net.tensors, net.vecs, pl2.d_w_sparse, v)
        want = forward(tokens.float(), full, vec, net.blocks, lambda h, t, i: h @ t.t())
    off = float((got - want).norm() / want.norm())
    one, many = float(losses[0]) if losses else float("nan"), float(losses[-1]) if losses else float("nan")
    kept = float(torch.count_nonzero(arena)) / net.n_weights
    print(f"{net.n_weights} weights, {kept:.3f} of them kept under the mask; loss {one:.4f} -> {many:.4f} in {a.steps} steps")
    print(f"dead channels per group {dead}; rebuilt {n_w} weights, {sum(m.q.numel() for m in served.w)} bytes of codes")
    print(f"8-bit output against the sparse network in fp32: {off:.4f} relative")
    result = dict(served=served, tokens=tokens, got=got, small=small, off=off, first=one, last=many, kept=kept, dead=dead, masked=[bool((t.detach()[m == 0] == 0).all())
                                                                              for t, m in zip(weights, masks)])
    torch.cuda.synchronize()
    pl.close()
    pl2.close()
    ops.close()
    return result


if __name__ == "__main__":
    main()
