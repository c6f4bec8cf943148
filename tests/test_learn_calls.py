"""Log probabilities, gradient norms and adapters without a GPU: what the calls refuse before anything is launched (host tensors are
refused as the last of a tensor's checks), how calls are shared out, and which tensors may be written."""
import os
import random
import subprocess

import pytest
import torch

from paper_2309_06973_amd import q8, shifter as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def calls():
    if not (os.path.exists(q8._CALLS_PATH) and os.path.exists(S._LIB_PATH)):
        from paper_2309_06973_amd import build
        build.build_library(verbose=False)
    return q8.load_calls()


X, T, V = torch.zeros(3, 8), torch.zeros(3, dtype=torch.int64), torch.zeros(3)
A, B = torch.zeros(2, 4, 8), torch.zeros(2, 8, 4)


def grad(*shape):
    return torch.ones(*shape, requires_grad=True)


REFUSED = [
    (lambda c: c.log_probs(0, 0, None, T, 1.0, False, 0, None), "tensor"),
    (lambda c: c.log_probs(0, 0, X.double(), T, 1.0, False, 0, None), "two-dimensional"),
    (lambda c: c.log_probs(0, 0, X[0], T, 1.0, False, 0, None), "two-dimensional"),
    (lambda c: c.log_probs(0, 0, X.t(), T, 1.0, False, 0, None), "side by side"),
    (lambda c: c.log_probs(0, 0, X, T, 1.0, False, 0, None), "cuda:0"),
    (lambda c: c.log_probs_grad(0, 0, X, T, V, V, None, None, None, 1.0, None), "cuda:0"),
    (lambda c: c.log_probs_grad(0, 0, grad(3, 8), T, V, V, None, None, None, 1.0, X), "needs a gradient"),
    (lambda c: c.log_probs_grad(0, 0, X, T, V, grad(3), None, None, None, 1.0, X), "needs a gradient"),
    (lambda c: c.grad_norm(0, 0, 5, None, 1.0, None, None), None),
    (lambda c: c.grad_norm(0, 0, [X], [], 1.0, None, None), "an entry for each"),
    (lambda c: c.grad_norm(0, 0, [X], None, 1.0, [], None), "an entry for each"),
    (lambda c: c.grad_norm(0, 0, [X], None, -1.0, None, None), "negative"),
    (lambda c: c.grad_norm(0, 0, [X], None, float("nan"), None, None), "negative"),
    (lambda c: c.grad_norm(0, 0, [X.double()], None, 1.0, None, None), "fp32, bf16 or fp16"),
    (lambda c: c.grad_norm(0, 0, [T], None, None, None, None), "fp32, bf16 or fp16"),
    (lambda c: c.grad_norm(0, 0, [X.to_sparse()], None, None, None, None), "fp32, bf16 or fp16"),
    (lambda c: c.grad_norm(0, 0, [X[:, :3]], None, None, None, None), "gaps"),
    (lambda c: c.grad_norm(0, 0, [X[:1].expand(3, 8)], None, None, None, None), "gaps"),
    (lambda c: c.grad_norm(0, 0, [None], None, None, None, None), "tensor"),
    (lambda c: c.grad_norm(0, 0, [grad(3)], None, None, None, None), "needs a gradient"),
    (lambda c: c.grad_norm(0, 0, [X], None, None, None, None), "cuda:0"),
    (lambda c: c.adapters(0, 0, X, X, A.double(), B, T, None, None, None, None), "a must be"),
    (lambda c: c.adapters(0, 0, X, X, A[0], B, T, None, None, None, None), "a must be"),
    (lambda c: c.adapters(0, 0, X, X, A.transpose(1, 2), B, T, None, None, None, None), "a must be"),
    (lambda c: c.adapters(0, 0, X, X, A, B[:1], T, None, None, None, None), "b must be"),
    (lambda c: c.adapters(0, 0, X, X, A, B.half(), T, None, None, None, None), "b must be"),
    (lambda c: c.adapters(0, 0, X, X, A, B, T, None, None, None, None), "cuda:0"),
    (lambda c: c.adapters(0, 0, X, X, grad(2, 4, 8), B, T, None, X, None, None), "needs a gradient"),
    (lambda c: c.adapters(0, 0, grad(3, 8), X, A, B, T, None, X, None, None), "needs a gradient"),
    (lambda c: c.adapters_grad(0, 0, X, X, A, B, T, None, None, True, None), "cuda:0"),
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_refusals(calls, i):
    call, what = REFUSED[i]
    with pytest.raises((ValueError, TypeError), match=what):
        call(calls)


@pytest.mark.parametrize("name, n", [("log_probs", 8), ("log_probs_grad", 11), ("grad_norm", 7), ("adapters", 11), ("adapters_grad", 11)])
def test_numbers_of_arguments(calls, name, n):
    for count in (0, n - 1, n + 1):
        with pytest.raises(TypeError):
            getattr(calls, name)(*([0] * count))
    with pytest.raises(TypeError):
        getattr(calls, name)(*(["no handle"] * n))


def test_the_c_interface_without_a_context(calls):
    lib = S.load_library()
    assert lib.shifter_log_probs(None, None) == S.SHIFTER_ERR_INVALID_ARG
    assert lib.shifter_log_probs(None, S.C.byref(S.LogProbsArgs())) == S.SHIFTER_ERR_INVALID_ARG
    assert lib.shifter_log_probs_grad(None, S.C.byref(S.LogProbsGradArgs())) == S.SHIFTER_ERR_INVALID_ARG
    assert lib.shifter_grad_norm(None, None, 0, None, None, 0) == S.SHIFTER_ERR_INVALID_ARG
    assert lib.shifter_clip_grad_norm(None, None, 0, 1.0, None, None, 0) == S.SHIFTER_ERR_INVALID_ARG
    assert lib.shifter_adapters(None, S.C.byref(S.AdaptersArgs())) == S.SHIFTER_ERR_INVALID_ARG
    assert lib.shifter_adapters_grad(None, S.C.byref(S.AdaptersGradArgs())) == S.SHIFTER_ERR_INVALID_ARG
    for call in (lambda: lib.shifter_log_probs_layout(1, 1, 0, None), lambda: lib.shifter_grad_norm_layout(1, None),
                 lambda: lib.shifter_adapters_layout(1, 1, 1, 1, 1, None), lambda: lib.shifter_adapters_grad_layout(1, 1, 1, 1, 1, 0, None)):
        assert call() == S.SHIFTER_ERR_INVALID_ARG
    for call, what in ((lambda: S.shifter_log_probs_layout(1, 40, 33), "32 alternatives"), (lambda: S.shifter_log_probs_layout(1, 4, 5), "than columns"),
                       (lambda: S.shifter_log_probs_layout(1 << 31, 4, 0), "2\\^31"), (lambda: S.shifter_grad_norm_layout(1 << 32), "2\\^32"),
                       (lambda: S.shifter_adapters_layout(1, 1, 1, 0, 1), "1 to 128"), (lambda: S.shifter_adapters_layout(1, 1, 1, 129, 1), "1 to 128"),
                       (lambda: S.shifter_adapters_layout((1 << 25) + 1, 1, 1, 1, 1), "2\\^25"), (lambda: S.shifter_adapters_layout(1, 1, 1, 1, 1 << 25), "2\\^24"),
                       (lambda: S.shifter_adapters_grad_layout(1, 1, 1, 1, 1, 3), "element type")):
        with pytest.raises(S.ShifterError, match=what):
            call()


def test_structures_are_as_in_the_header(tmp_path):
    names = dict(LogProbsArgs="shifter_log_probs_args", LogProbsGradArgs="shifter_log_probs_grad_args", Grad="shifter_grad", AdaptersArgs="shifter_adapters_args",
                 AdaptersGradArgs="shifter_adapters_grad_args")
    lines = [f'printf("{c}.{f[0]} %zu\\n", offsetof({h}, {f[0]}));' for c, h in names.items() for f in getattr(S, c)._fields_]
    lines += [f'printf("{c} %zu\\n", sizeof({h}));' for c, h in names.items()]
    (tmp_path / "s.c").write_text('#include <stddef.h>\n#include <stdio.h>\n#include "shifter.h"\nint main() {' + "\n".join(lines) + "return 0; }\n")
    subprocess.run(["gcc", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")], check=True)
    for line in subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.splitlines():
        name, at = line.split()
        c, _, field = name.partition(".")
        assert int(at) == (getattr(getattr(S, c), field).offset if field else S.C.sizeof(getattr(S, c))), name


PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include "adapters_plan.h"
#include "grad_norm_plan.h"
using namespace shifter;
typedef unsigned long long u;
int main(int n, char** v) {
    auto at = [&](int i) { return strtoull(v[i], 0, 10); };
    switch (v[1][0]) {
        case 'l': for (int i = 2; i + 2 < n; i += 3) {
            const LogProbsPlan p = log_probs_plan(at(i), at(i + 1), (uint32_t)at(i + 2));
            printf("%u %u %u %llu\n", p.threads, p.parts, p.part_cols, (u)p.bytes);
        } break;
        case 'g': {                              // elements of tensors: each tensor's chunks, then the list's
            std::vector<shifter_grad> all;
            for (int i = 2; i < n; ++i) all.push_back({(void*)(0x123456789000ull + 0x1000ull * i), (void*)0x2000, nullptr, at(i), i % 3});
            for (uint64_t from = 0; from < all.size(); from += GRAD_LIST) {
                GradList l;
                grad_list(all, from, GRAD_CHUNK, &l);
                for (uint32_t i = 0; i < l.n; ++i)
                    printf("%llu %u %u %u\n", (u)l.high[0][i] << 32 | l.low[0][i], l.first[i], (l.last[i] & 8191u) + 1u, l.last[i] >> 13);
                printf("%u\n", l.chunks);
            }
            printf("%d\n", (int)grad_small(all));
        } break;
        case 'o': {                              // g, out, elements of fp32 tensors: whether they overlap
            std::vector<shifter_grad> all;
            for (int i = 2; i + 2 < n; i += 3) all.push_back({(void*)at(i), (void*)at(i + 1), nullptr, at(i + 2), SHIFTER_F32});
            printf("%d\n", (int)grad_overlap(all));
        } break;
        case 'e': for (int i = 2; i + 6 < n; i += 7) // rows, columns of y, of x, x's stride, rank, adapters, bytes of an element
            printf("%d %u\n", (int)adapt_one(at(i), at(i + 2), at(i + 3), (uint32_t)at(i + 4), at(i + 5), at(i + 6)), adapt_one_blocks(at(i), at(i + 1), at(i + 5)));
        break;
        case 'a': for (int i = 2; i + 4 < n; i += 5) {
            const uint64_t m = at(i), nn = at(i + 1), k = at(i + 2), many = at(i + 4);
            const uint32_t rank = (uint32_t)at(i + 3);
            bool c;
            if (adapters_bad_sizes(m, nn, k, rank, many, &c)) { printf("bad\n"); continue; }
            const AdaptersPlan p = adapters_plan(m, k, rank, many);
            const AdaptersGradPlan q = adapters_grad_plan(m, nn, k, rank, many, 2);
            printf("%u %llu %u %u %u %llu %u %u %u %u %u %llu %llu %llu %llu %llu %llu %llu %llu\n", p.parts, (u)p.bytes, adapt_tiles(m, rank), adapt_jobs(m, many),
                   adapt_down_jobs(m, many), (u)p.order, (unsigned)adapt_sorted(m, many), q.parts_x, q.parts_g, q.parts_rows, q.rows_each, (u)q.down, (u)q.up, (u)q.sums,
                   (u)q.a, (u)q.b, (u)q.rows, (u)q.partial, (u)q.bytes);
        } break;
    }
    return 0;
}
"""
up = lambda a, b: -(-a // b)


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    where = tmp_path_factory.mktemp("learn")
    (where / "plan.cpp").write_text(PROGRAM)
    exe = str(where / "plan")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2309_06973_amd", "csrc"), "-I", os.path.join(ROOT, "include"),
                    str(where / "plan.cpp"), "-o", exe], check=True)

    def ask(kind, numbers):
        return subprocess.run([exe, kind] + [str(x) for x in numbers], capture_output=True, text=True, check=True).stdout.splitlines()
    return ask


def test_parts_of_rows_of_logits(plan):
    rng = random.Random(2)
    sizes = [(int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 25)), rng.choice([0, 1, 8, 9, 32])) for _ in range(1500)]
    shared = 0
    for (rows, cols, top), line in zip(sizes, plan("l", [x for s in sizes for x in s])):
        threads, parts, part_cols, size = map(int, line.split())
        assert part_cols % 8 == 0 and (parts - 1) * part_cols < cols <= parts * part_cols and parts <= 64
        assert threads == 256 or (parts == 1 and cols <= {16: 256, 64: 1024}[threads])
        if parts == 1:
            assert size == 0
        else:
            shared += 1
            assert rows < 512 and 4 * rows <= S.SHIFTER_LEARN_ZERO and size >= S.SHIFTER_LEARN_ZERO + rows * parts * (16 + 8 * top)
            # the best few of each part are enough for a bound of the top
            assert parts * min(top, 64 // parts) >= top
    assert shared > 100


def test_lists_of_gradients(plan):
    rng = random.Random(3)
    sizes = [int(2 ** rng.uniform(0, 24)) for _ in range(400)] + [2048, 2049, 4096, 1]
    lines = plan("g", sizes)
    at, first = 0, 0
    for i, n in enumerate(sizes):
        address, start, last, dtype = map(int, lines[at].split())
        assert address == 0x123456789000 + 0x1000 * (i + 2) and start == first and dtype == (i + 2) % 3 and last == (n - 1) % 2048 + 1
        first += up(n, 2048)
        at += 1
        if (i + 1) % 164 == 0 or i + 1 == len(sizes):
            assert int(lines[at]) == first
            first, at = 0, at + 1
    assert int(lines[at]) == 0
    assert plan("g", [32760])[-1] == "1" and plan("g", [32768])[-1] == "1" and plan("g", [32769])[-1] == "0" and plan("g", [8] * 164)[-1] == "1"
    assert plan("g", [8] * 165)[-1] == "0" and plan("g", [1 << 36])[-1] == "0" and plan("g", [1] * 100 + [31968])[-1] == "1"


def test_tensors_that_overlap(plan):
    """Against the definition: two spans meet, and one of them is written; a tensor's own elements in place do not count."""
    rng = random.Random(4)
    seen = [0, 0]
    for _ in range(300):
        many = rng.randint(1, 6)
        spread = rng.choice([200, 2000])
        grads = []
        for _ in range(many):
            g = 4 * rng.randint(1, spread)
            grads.append((g, g if rng.random() < 0.5 else 4 * rng.randint(1, spread), rng.randint(1, 40)))
        spans = [(i, o, o + 4 * n, True) for i, (g, o, n) in enumerate(grads)] + [(i, g, g + 4 * n, False) for i, (g, o, n) in enumerate(grads) if g != o]
        want = any((a[3] or b[3]) and a[1] < b[2] and b[1] < a[2] for x, a in enumerate(spans) for b in spans[x + 1:])
        assert int(plan("o", [v for e in grads for v in e])[0]) == want
        seen[want] += 1
    assert min(seen) > 50


def test_adapters_in_one_launch(plan):
    rng = random.Random(6)
    size = lambda most: int(2 ** rng.uniform(0, most))
    sizes = [(size(8), size(14), size(12), rng.randint(0, 8), rng.randint(1, 40), rng.choice([0, 1, 7, 8, 64]), rng.choice([2, 4])) for _ in range(2000)]
    sizes += [(m, n, 4096, 0, 16, 8, 2) for m in (1, 2, 3, 16, 128, 129) for n in (0, 1, 256, 257, 4096, 1 << 31)]
    sizes = [(m, n, k // 8 * 8 if i % 2 else k, k + gap, rank, many, b) for i, (m, n, k, gap, rank, many, b) in enumerate(sizes)]
    seen = [0, 0]
    for (m, n, k, ld, rank, many, b), line in zip(sizes, plan("e", [x for s in sizes for x in s])):
        one, blocks = map(int, line.split())
        # whole pieces of eight of A and x, and not many of them
        assert one == (m <= 128 and rank <= 32 and many > 0 and k % 8 == 0 and ld % 8 == 0 and (rank + min(m, 16)) * k * b <= 147456)
        assert 1 <= blocks <= max(1, up(n, 256)) and blocks * up(m, 16) * (1 if m > 128 else max(1, min(16, m, many))) <= max(256, up(m, 16) * 16)
        seen[one] += 1
    assert min(seen) > 50


def test_adapters_workspaces(plan):
    rng = random.Random(5)
    size = lambda most: int(2 ** rng.uniform(0, most))
    sizes = [(size(20), size(14), size(14), rng.randint(1, 128), rng.choice([1, 2, 7, 8, 64, 500])) for _ in range(1500)]
    sizes += [(m, 4096, 4096, 16, a) for m in (1, 16, 127, 128, 129, 256, 2047, 2048, 8192) for a in (1, 7, 8, 4094, 4095)]
    for (m, n, k, rank, many), line in zip(sizes, plan("a", [x for s in sizes for x in s])):
        if line == "bad":
            assert many * (1 + up(k, 64) + up(n, 64)) >= 1 << 24
            continue
        parts, total, tiles, jobs, down_jobs, order, ordered, px, pg, pr, each, down, over, sums, a, b, rows, partial, everything = map(int, line.split())
        pad = up(rank, 16) * 16
        assert order >= parts * m * pad * 4 and total >= order + (4 * m if ordered else 0) and 1 <= parts <= (32 if m <= 128 else 2)
        assert parts <= max(1, up(k, 64)) and px == parts and ordered == (m > 128 and 8 <= many <= 4094)
        # a tile of few rows: no more adapters than blocks that share it
        assert jobs == (1 if m > 128 else max(1, min(16, m, many))) and (m > 128 or down_jobs == jobs) and tiles in (1, 2)
        assert (tiles == 1 or rank <= 32) and up(m, 16 * tiles) * 256 < 1 << 32
        assert each % 16 == 0 and pr == max(1, up(m, each)) and pr <= 16
        # pieces one behind the other
        need = [(down, m * pad * 4), (over, m * pad * 4), (sums, max(px, pg) * m * pad * 4), (a, many * k * rank * 2), (b, many * n * rank * 2), (rows, 4 * m)]
        for (x, bytes_), (y, _) in zip(need, need[1:] + [(partial, 0)]):
            assert x % 256 == 0 and x + bytes_ <= y
        assert partial + ((pr + many) * (k + n) * rank * 4 if pr > 1 else 0) <= everything
        # an adapter's parts have places of their own, for any shares of the rows
        shares = sorted(rng.randint(0, m) for _ in range(many - 1)) if many < 100 else []
        first = [0] + shares + [m]
        used = set()
        for i in range(len(first) - 1):
            for p in range(up(first[i + 1] - first[i], each)):
                place = first[i] // each + i + p
                assert place not in used and place < pr + many
                used.add(place)
