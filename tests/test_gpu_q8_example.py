"""The example that runs the 8-bit operators together: a residual network pruned, trained on under its
mask with 8-bit checkpoints, rebuilt, and served in 8 bits.

The served output is compared with the same network worked out from the operators' definition in 64 bits:
quantised weights and biases, codes, whole-number sums, bf16 where the example holds bf16.  The two
differ where a 64-bit value and the library's 32-bit one lie on different sides of a rounding to bf16:
by one step of it, 2^-7 at most and 2^-8 on average, for some of the values of each of the
2 b + 2 products and b additions.  Were it all of them, the output would be off by (3 b + 2) 2^-8 of
its norm: that is allowed."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import q8_oracle as Q

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("residual_mlp_q8", os.path.join(ROOT, "examples", "residual_mlp_q8.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def served_by_definition(served, w, tokens):
    """Served.__call__ on the CPU, from the rebuilt weights."""
    held = lambda c: torch.from_numpy(c).to(torch.bfloat16)
    weights = [Q.quantize(t) for t in w]
    product = lambda x, i, bias=None: Q.product(*x, *weights[i], None if bias is None else Q.f64(bias))[0]
    eps = float(np.float32(served.eps))
    h, added = held(product(Q.quantize(tokens), 0)), None
    for b in range(served.blocks):
        q, s, h = Q.rms_norm(h, served.norms[b], eps, added)
        u = held(product((q, s), 1 + 2 * b, served.biases[b]))
        added = held(product(Q.quantize(u, relu=True), 2 + 2 * b))
    q, s, _ = Q.rms_norm(h, served.norms[-1], eps, added)
    return product((q, s), len(w) - 1)


@pytest.mark.parametrize("blocks,args", [(3, ["--steps", "10"]), (2, ["--stream", "200", "--hidden", "333", "--tokens", "7", "--steps", "5"]),
                                         (1, ["--tokens", "1", "--steps", "3", "--sparsity", "0.5"])])
def test_example(blocks, args, capsys):
    r = example().main(["--blocks", str(blocks)] + args)
    want = served_by_definition(r["served"], r["small"][0], r["tokens"])
    got = Q.f64(r["got"])
    assert np.linalg.norm(got - want) <= (3 * blocks + 2) * 2.0 ** -8 * np.linalg.norm(want)
    assert r["last"] < r["first"]
    assert all(r["masked"])                       # no pruned weight came back
    assert sum(r["dead"]) > 0                     # the rebuild had channels to remove
    assert "relative" in capsys.readouterr().out
