"""The ends of the numbers on every way that the weight gradient can take: columns of zeros, of the smallest and the largest
numbers side by side, one row far above the others, values that are not finite, sums added to what there is.

Which way a size takes is asked of the header, on the host.  The bound is the one that the interface states, per entry
(q8_oracle.weight_grad); p below the normal numbers is held in steps of 2^-149, which adds half of one a term (a whole one
is allowed); adding to what there is rounds once."""
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import q8_oracle as Q
from paper_2309_06973_amd.q8 import Q8
from test_gpu_q8_product import check_gradient, grads, matrix

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda"
# one launch in 64 bits; few rows of a large result; digits in one launch by 256, 512 and 1024 threads; digits in slices, rows in
# parts and not
WAYS = {"small": (200, 70, 45), "few rows": (16, 1100, 1000), "256": (300, 1100, 1000), "512": (700, 1100, 1001), "1024": (1500, 1060, 1010),
        "slices, parts": (2500, 70, 45), "slices, many parts": (20000, 70, 51), "slices": (2500, 2300, 2047)}

PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include "q8_plan.h"
int main(int n, char** v) {
    for (int i = 1; i + 2 < n; i += 3) {
        const uint64_t m = strtoull(v[i], 0, 10);
        const shifter::Q8GradientPlan g = shifter::q8_gradient_plan(m, strtoull(v[i + 1], 0, 10), strtoull(v[i + 2], 0, 10));
        printf("%d %u %u %llu\n", (int)g.kernel, g.parts, g.slices, (unsigned long long)g.ld);
    }
    return 0;
}
"""


def test_the_ways(tmp_path):
    src = tmp_path / "ways.cpp"
    src.write_text(PROGRAM)
    exe = str(tmp_path / "ways")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2309_06973_amd", "csrc"),
                    str(src), "-o", exe], check=True)
    out = subprocess.run([exe] + [str(x) for s in WAYS.values() for x in s], capture_output=True, text=True, check=True).stdout
    got = dict(zip(WAYS, (tuple(map(int, l.split())) for l in out.splitlines())))
    assert got["small"][0] == -1 and got["few rows"][0] == -2
    assert all(got[w][0] >= 0 and got[w][2] == 0 for w in ("256", "512", "1024"))
    assert got["256"][3] <= 512 < got["512"][3] <= 1024 < got["1024"][3]
    assert all(got[w][0] >= 0 and got[w][2] > 0 for w in WAYS if "slices" in w)
    assert 1 < got["slices, parts"][1] < got["slices, many parts"][1] and got["slices"][1] == 1


@pytest.fixture(scope="module")
def ops():
    o = Q8()
    yield o
    torch.cuda.synchronize()
    o.close()


def steps(q):
    """What p in steps of 2^-149 adds to the bound."""
    return (2.0 ** -149 * np.abs(q.astype(np.float64)).sum(0))[None, :]


@pytest.mark.gpu
@pytest.mark.parametrize("way", WAYS)
def test_magnitudes(ops, way):
    m, n, k = WAYS[way]
    e = torch.linspace(-135, 100, n, dtype=torch.float64)
    g = (torch.randn(m, n, dtype=torch.float64, generator=torch.Generator().manual_seed(1)) * 2.0 ** e).float()
    g[:, 5] = 0
    g[:, n - 1] = 0
    g[m // 3] *= 2.0 ** 14
    g = g.to(DEV)
    x, q, s = matrix(m, k, 7)
    x.scale[m // 4:m // 3 - 1] = 0
    s[m // 4:m // 3 - 1] = 0
    got = ops.weight_grad(g, x)
    want, bound = Q.weight_grad(g, q, s)
    assert (np.abs(Q.f64(got) - want) <= 1.001 * (bound + steps(q))).all()
    assert (got[5] == 0).all() and (got[n - 1] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("far", [1e4, 1e6])
def test_a_row_far_above_the_others(ops, way, far):
    """Behind a ReLU, so that half of the entries have nothing of that row."""
    m, n, k = WAYS[way]
    g = grads(m, n, "fp32", 3)
    g[m // 2] *= far
    x, q, s = matrix(m, k, 5)
    x.q[x.q < 0] = 0
    q = np.maximum(q, 0)
    want, bound = Q.weight_grad(g, q, s)
    assert (np.abs(Q.f64(ops.weight_grad(g, x)) - want) <= 1.001 * bound).all()


@pytest.mark.gpu
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_not_finite(ops, way, value):
    m, n, k = WAYS[way]
    x, q, s = matrix(m, k, 3)
    x.q[m - 1, :16] = 0                        # codes that an infinity meets as 0 and not
    g = grads(m, n, "bf16", 4)
    clean = ops.weight_grad(g, x)
    assert torch.isfinite(clean).all()
    g[m - 1, 66] = value
    mask = torch.ones((n, k), dtype=torch.uint8, device=DEV)
    mask[66, 5] = 0
    for accumulate in (False, True):
        old = torch.ones((n, k), device=DEV)
        d = ops.weight_grad(g, x, mask=mask, out=old.clone(), accumulate=accumulate)
        assert torch.isnan(d[66][mask[66] != 0]).all() and d[66, 5] == float(accumulate)
        others = torch.arange(n, device=DEV) != 66
        assert torch.equal(d[others], clean[others] + 1.0 if accumulate else clean[others])
    x.scale[m // 2] = float("nan")             # a token that could not be coded: every column has it
    assert torch.isnan(ops.weight_grad(g, x)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_added_under_a_mask(ops, way, dtype):
    m, n, k = WAYS[way]
    check_gradient(ops, m, n, k, dtype, seed=m, mask=True, accumulate=True, gap=1, shift=1)
    check_gradient(ops, m, n, k, dtype, seed=m + 1, accumulate=True)
