"""Every tile of the 8-bit product and gradient at sizes that take it: whole tiles, tiles that end inside, as
many stages as its buffers hold and one more or less, rows split into parts.  Which kernel a size takes
is asked of the header itself, on the host.  Tolerances as in test_gpu_q8_product.py."""
import os
import subprocess

import pytest
import torch

from paper_2309_06973_amd.q8 import Q8
from test_gpu_q8_product import check_gradient, check_product

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PRODUCT = {"few": [(1, 40, 8192), (16, 4096, 8200), (5, 100, 12289), (9, 64, 4095), (16, 33, 3000), (1, 20, 1025), (1, 20, 2049),
                   (1, 20, 3100), (17, 300, 2049), (30, 70, 4097), (48, 129, 3541), (40, 16, 6145)],
           "groups": [(100, 500, 8200), (128, 640, 512), (65, 257, 513), (300, 129, 640), (500, 300, 2000), (2000, 64, 4001), (12000, 16, 100),
                      (49, 1000, 127), (50, 2040, 1), (4000, 33, 260), (5000, 17, 9000)],
           "64x64": [(256, 1024, 127), (300, 1000, 640), (257, 1023, 513), (512, 640, 385)],
           "64x128": [(512, 4096, 384), (512, 4096, 385), (777, 2900, 400), (640, 3500, 130), (1000, 2500, 513)],
           "128x128": [(2000, 1990, 1300), (1100, 3541, 2100), (1024, 4096, 1500)],
           "128x256": [(2048, 4096, 1025), (1999, 4090, 2100), (2040, 4096, 700), (4096, 4096, 513)],
           "256x256": [(4000, 4090, 1500), (4081, 3900, 1900)]}
GRADIENT = {"64x64": [(700, 1500, 1000), (2047, 1500, 700), (1300, 1999, 900), (129, 4097, 1023)],
            "64x64 deep": [(256, 2048, 512), (150, 1000, 1000), (3000, 500, 400), (20000, 60, 50), (1025, 513, 700)],
            "64x128": [(512, 4096, 1024), (300, 3000, 1500), (1500, 2000, 2049)],
            "64x128 deep": [(2048, 1873, 977), (1700, 1900, 1000), (2047, 1900, 1024)],
            "64x256": [(2048, 2048, 2048), (1800, 2000, 2047)],
            "128x256": [(2500, 4000, 2047)]}

PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include "q8_plan.h"
int main(int n, char** v) {
    using namespace shifter;
    for (int i = 1; i + 3 < n; i += 4) {
        const uint64_t a = strtoull(v[i + 1], 0, 10), b = strtoull(v[i + 2], 0, 10), c = strtoull(v[i + 3], 0, 10);
        if (v[i][0] == 'p') printf("%d 1\n", (int)q8_kernel_for(a, b, c));
        else { const Q8GradientPlan g = q8_gradient_plan(a, b, c); printf("%d %u\n", (int)g.kernel, g.parts); }
    }
    return 0;
}
"""


def test_sizes_take_their_kernels(tmp_path):
    src = tmp_path / "plan.cpp"
    src.write_text(PROGRAM)
    exe = str(tmp_path / "plan")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2309_06973_amd", "csrc"),
                    str(src), "-o", exe], check=True)
    cases = [("p", i, s) for i, v in enumerate(PRODUCT.values()) for s in v] + \
            [("g", i, s) for i, v in enumerate(GRADIENT.values()) for s in v]
    out = subprocess.run([exe] + [str(x) for kind, _, s in cases for x in (kind, *s)], capture_output=True, text=True, check=True)
    got = [tuple(map(int, l.split())) for l in out.stdout.splitlines()]
    wrong = [(c, g) for c, g in zip(cases, got) if c[1] != g[0]]
    assert not wrong, wrong
    assert any(g[1] > 1 for c, g in zip(cases, got))                 # rows split into parts


@pytest.fixture(scope="module")
def ops():
    o = Q8()
    yield o
    torch.cuda.synchronize()
    o.close()


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [s for v in PRODUCT.values() for s in v])
def test_product_tiles(ops, m, n, k):
    check_product(ops, m, n, k, "bf16", seed=m + n + k, bias=True, ends=k % 2 == 1)


@pytest.mark.gpu
@pytest.mark.parametrize("k", [0, 1, 3, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 500, 1000])
def test_product_tile_sums(ops, k):
    check_product(ops, 300 + k % 7, 1000 + k % 5, k, "fp32", seed=k, bias=True, relu=k % 2 == 0, gap=k % 3, extra=16 * (k % 2))


@pytest.mark.gpu
@pytest.mark.parametrize("e", [0, 1, 15, 16, 17, 31, 33, 63])
def test_product_tile_edges(ops, e):
    check_product(ops, 320 + e, 960 + e, 200, "bf16", seed=e, gap=e % 3)
    check_product(ops, 513 - e, 2049 - e, 130, "fp16", seed=e, bias=True)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [s for v in GRADIENT.values() for s in v])
def test_gradient_tiles(ops, m, n, k):
    check_gradient(ops, m, n, k, "bf16", seed=m + n + k, mask=True, accumulate=k % 2 == 1, gap=m % 2)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [100, 511, 512, 513, 700, 1023, 1024, 1025, 1537, 2047, 2048, 2049])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_digits(ops, m, dtype):
    """Digits of all rows at once by 256, 512 and 1024 threads, and in slices."""
    check_gradient(ops, m, 1060, 1010, dtype, seed=m, gap=m % 3, shift=m % 2)
    check_gradient(ops, m, 5, 300, dtype, seed=m)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (3, 15, 17), (15, 16, 32), (16, 17, 33), (17, 33, 31), (63, 64, 1), (127, 1, 64), (128, 49, 50),
                                   (129, 100, 100), (1000, 90, 70), (1024, 362, 361), (2048, 256, 255), (2047, 257, 250), (300, 256, 256), (300, 257, 256), (64, 1024, 1024), (40, 1500, 690), (5, 997, 1050),
                                   (2, 1100, 1000), (16, 1030, 1025), (7, 4, 300000), (13, 300000, 4)])
def test_little_work(ops, m, n, k, dtype):
    """One launch in 64 bits: both widths of its blocks, and few rows of a large result."""
    check_gradient(ops, m, n, k, dtype, seed=m + n + k)
    check_gradient(ops, m, n, k, dtype, seed=m + n + k, mask=True, accumulate=True, gap=1 + m % 2, shift=1)


@pytest.mark.gpu
def test_recorded_workspace():
    """A recorded gradient keeps its workspace to itself: replays on another stream than the handle's, with calls made at once
    of other sizes under way beside them, give what they gave alone."""
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ops = Q8()
        gen = torch.Generator(device="cuda").manual_seed(5)
        rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
        g, x = rand(2700, 300), ops.quantize(rand(2700, 200))
        g2, x2 = rand(2900, 310), ops.quantize(rand(2900, 190))
        want, want2 = ops.weight_grad(g, x), ops.weight_grad(g2, x2)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            recorded = ops.weight_grad(g, x)
        assert len(ops.recorded) == 1 and ops.recorded[0].data_ptr() != ops.work.data_ptr()
        torch.cuda.synchronize()
        for _ in range(20):
            recorded.zero_()
            other.wait_stream(stream)
            with torch.cuda.stream(other):
                graph.replay()
            got2 = ops.weight_grad(g2, x2)
            torch.cuda.synchronize()
            assert torch.equal(recorded, want) and torch.equal(got2, want2)
        ops.close()


@pytest.mark.gpu
def test_no_rows_of_a_large_result(ops):
    g, x = torch.zeros((0, 1100), device="cuda"), ops.quantize(torch.zeros((0, 1000), device="cuda"))
    assert (ops.weight_grad(g, x) == 0).all()
    old = torch.randn((1100, 1000), device="cuda")
    assert torch.equal(ops.weight_grad(g, x, out=old.clone(), accumulate=True), old)
