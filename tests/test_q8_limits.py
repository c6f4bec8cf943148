"""Which sizes the 8-bit product and gradient refuse as more than a launch holds: the header's checks on the host
against grids worked out here, the layout call, and on the device the sizes next to them."""
import os
import random
import subprocess

import pytest
import torch

from paper_2309_06973_amd import shifter as S
from paper_2309_06973_amd.q8 import Q8, Q8Matrix

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include "q8_plan.h"
using namespace shifter;
int main(int n, char** v) {
    for (int i = 1; i + 2 < n; i += 3) {
        const uint64_t a = strtoull(v[i], 0, 10), b = strtoull(v[i + 1], 0, 10), c = strtoull(v[i + 2], 0, 10);
        const bool product = !q8_too_many(a, b), gradient = !q8_gradient_too_many(a, b, c);
        Q8GradientPlan g{};
        if (gradient) g = q8_gradient_plan(a, b, c);
        printf("%d %d %d %d %u %llu\n", product, product ? (int)q8_kernel_for(a, b, c) : 0, gradient, gradient ? (int)g.kernel : 0, g.parts,
               (unsigned long long)g.bytes);
    }
    return 0;
}
"""
LAUNCH = 1 << 32                       # threads along an axis
up = lambda a, b: -(-a // b)


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    where = tmp_path_factory.mktemp("q8")
    src = where / "limits.cpp"
    src.write_text(PROGRAM)
    exe = str(where / "limits")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2309_06973_amd", "csrc"),
                    str(src), "-o", exe], check=True)

    def ask(sizes):
        out = subprocess.run([exe] + [str(x) for s in sizes for x in s], capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, l.split())) for l in out.splitlines()]
    return ask


# rows, columns and threads of a block: few rows, groups of them, then the tiles
PRODUCT = [(48, 16, 1024), (16, 16, 1024), (64, 64, 256), (64, 128, 512), (128, 128, 512), (128, 256, 512), (256, 256, 512)]
GRADIENT = {-2: (16, 256, 256), -1: (16, 16, 512), 0: (64, 64, 256), 1: (64, 64, 256), 2: (64, 128, 512), 3: (64, 128, 512), 4: (64, 256, 512),
            5: (128, 256, 512)}


def test_what_is_accepted_fits_a_launch(plan):
    rng = random.Random(1)
    size = lambda most: max(1, int(2 ** rng.uniform(0, most)))
    sizes = [(size(30.99), size(30.99), size(16.99)) for _ in range(1500)] + [(size(17), size(30.99), size(22)) for _ in range(2500)]
    accepted = [0, 0]
    for (m, n, k), (product, kernel, gradient, tiles, parts, size) in zip(sizes, plan(sizes)):
        if product:
            accepted[0] += 1
            rows, cols, threads = PRODUCT[kernel]
            assert (up(n, cols) if kernel < 2 else up(m, rows) * up(n, cols)) * threads < LAUNCH, (m, n, k)
        if not gradient or m > S.SHIFTER_Q8_MAX_SUM:
            continue
        accepted[1] += 1
        rows, cols, threads = GRADIENT[tiles]
        assert up(n, rows) * up(k, cols) * threads < LAUNCH and parts <= 32, (m, n, k)
        if tiles < 0:
            assert size == 0
            continue
        ld = up(m, 128) * 128
        # largest of the columns in slices, three planes of digits, codes, sums of the parts
        assert size >= 3 * n * ld + k * ld + (4 * parts * n * k if parts > 1 else 0) and size < 1 << 50
        if m <= 2048:
            threads = 256 if ld <= 512 else 512 if ld <= 1024 else 1024
            assert (up(n, 16) + up(up(k, 128) * (ld // 128), threads // 256)) * threads < LAUNCH, (m, n, k)
        else:
            slices = up(m, 32 * up(m, 4096))
            deep = min(8, max(1, up(n, 64) * (ld // 128) // 2048))
            assert (up(n, 512) * slices + up(k, 128) * (ld // 128)) * 256 < LAUNCH, (m, n, k)
            assert up(n, 64) * up(ld // 128, deep) * 256 < LAUNCH, (m, n, k)
    assert min(accepted) > 500, accepted


def test_what_fits_a_launch_is_accepted(plan):
    """Narrow results of many rows, and of many columns: the product has no blocks of 256 columns."""
    sizes = [(1 << 28, 1, 16), (1 << 28, 64, 16), ((1 << 29) - 64, 1, 16), (1 << 29, 1, 16), (64, 1 << 26, 16), (49, (1 << 29) - 64, 16),
             (16, (1 << 26) - 16, 16), (16, (1 << 26) - 15, 16)]
    assert [p[0] for p in plan(sizes)] == [1, 1, 1, 0, 1, 1, 1, 0]
    sizes = [(0, 1, (1 << 31) - 1), (16, (1 << 28) - 16, 256), (16, 1 << 28, 256), (17, (1 << 28) - 64, 64), (17, 1 << 28, 64), (300, 1, 1 << 22),
             (1000, 1 << 20, 1), (1000, 1 << 25, 1)]
    assert [p[2] for p in plan(sizes)] == [1, 1, 0, 1, 0, 1, 1, 1]


@pytest.mark.parametrize("m, n, k", [(17, (1 << 31) - 1, (1 << 31) - 1), (131071, (1 << 31) - 1, (1 << 31) - 1), (17, 1 << 29, 64),
                                     (16, 1 << 28, 256), (0, (1 << 31) - 1, (1 << 31) - 1)])
def test_the_layout_call_refuses_what_the_call_refuses(m, n, k):
    with pytest.raises(S.ShifterError, match="more tiles than a launch holds") as e:
        S.shifter_weight_grad_q8_layout(m, n, k)
    assert e.value.code == S.SHIFTER_ERR_CAPACITY


@pytest.mark.gpu
@pytest.mark.parametrize("m, n", [(1 << 28, 1), (64, 1 << 26)])
def test_long_narrow_products(m, n):
    """2^28 rows of one result, 2^26 columns of few: whole numbers up to 2^20, powers of two as scales, so fp32 holds them exactly."""
    ops, k = Q8(), 16
    g = torch.Generator(device="cuda").manual_seed(m)
    made = lambda rows: Q8Matrix(torch.randint(-128, 128, (rows, k), generator=g, device="cuda", dtype=torch.int8),
                                 torch.full((rows,), 0.5, device="cuda"), k)
    a, b = made(m), made(n)
    c = ops.matmul(a, b, dtype=torch.float32)
    step = 1 << 22
    for i in range(0, max(m, n), step):
        rows, cols = (slice(i, i + step), slice(None)) if m > n else (slice(None), slice(i, i + step))
        want = 0.25 * (a.q[rows].float() @ b.q[cols].float().t())
        assert torch.equal(c[rows, cols], want), i
    torch.cuda.synchronize()
    ops.close()
