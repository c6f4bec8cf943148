"""Which lists of gradients may be clipped: what is written lies over nothing that the call reads or writes elsewhere, masks
among it."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include "grad_norm_plan.h"
using namespace shifter;
int main() {                               // lists: their length, then g, out, mask, elements, type of each
    unsigned long long n, v[5];
    while (scanf("%llu", &n) == 1) {
        std::vector<shifter_grad> all;
        for (unsigned long long i = 0; i < n; ++i) {
            for (auto& x : v)
                if (scanf("%llu", &x) != 1) return 1;
            all.push_back({(void*)v[0], (void*)v[1], (const uint8_t*)v[2], v[3], (int)v[4]});
        }
        printf("%d\n", (int)grad_overlap(all));
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def overlap(tmp_path_factory):
    where = tmp_path_factory.mktemp("overlap")
    (where / "overlap.cpp").write_text(PROGRAM)
    exe = str(where / "overlap")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2309_06973_amd", "csrc"), "-I", os.path.join(ROOT, "include"),
                    str(where / "overlap.cpp"), "-o", exe], check=True)

    def ask(lists):
        text = "\n".join(" ".join(map(str, [len(l)] + [v for e in l for v in e])) for l in lists)
        return [line == "1" for line in subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split()]
    return ask


def meets(grads):
    """From the definition: two spans meet, and one of them is written; a tensor's own elements in place do not count."""
    spans = []
    for g, out, mask, n, dtype in grads:
        size = 4 if dtype == 0 else 2
        spans.append((out, out + size * n, True))
        if g != out:
            spans.append((g, g + size * n, False))
        if mask:
            spans.append((mask, mask + n, False))
    return any((a[2] or b[2]) and a[0] < b[1] and b[0] < a[1] for i, a in enumerate(spans) for b in spans[i + 1:])


def test_masks_among_them(overlap):
    rng = random.Random(4)
    lists = []
    for _ in range(3000):
        spread, many = rng.choice([100, 400, 4000]), rng.randint(1, 5)
        place = lambda: 4 * rng.randint(1, spread)
        one = []
        for _ in range(many):
            g = place()
            one.append((g, g if rng.random() < 0.5 else place(), rng.choice([0, place() + rng.randint(0, 3)]), rng.randint(1, 30), rng.randint(0, 2)))
        lists.append(one)
    got = overlap(lists)
    assert got == [meets(l) for l in lists]
    without = overlap([[(g, o, 0, n, t) for g, o, _, n, t in l] for l in lists])
    assert sum(got) > 300 and sum(not g for g in got) > 300 and sum(g and not w for g, w in zip(got, without)) > 100


def test_masks_that_lie_beside_or_over_each_other(overlap):
    free = [(1000, 2000, 3000, 100, 0), (5000, 5000, 3000, 100, 0)]                    # one mask for two
    beside = [(1000, 1000, 1400, 100, 0), (1500, 1500, 1400, 100, 0)]                  # [1400, 1500) between [1000, 1400) and [1500, 1900)
    into = [[(1000, 1000, 1399, 100, 0)], [(1000, 2000, 2399, 100, 0)], [(1000, 1000, 901, 100, 0)], [(1000, 2000, 1100, 100, 0)],
            [(1000, 1000, 0, 100, 1), (4000, 4000, 1199, 50, 2)], [(1000, 1000, 0, 100, 1), (4000, 4000, 1200, 50, 2)]]
    assert overlap([free, beside, *into]) == [False, False, True, True, True, False, True, False]
