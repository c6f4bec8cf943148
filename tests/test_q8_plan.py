"""8-bit matrices without a GPU: the checks of a call's arguments and the gradient's workspace
(the header compiled for the host), what the layout call refuses, what the Python layer refuses,
and the definition in 64 bits that the GPU tests go by."""
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import q8_oracle as Q
from paper_2309_06973_amd import shifter as S
from paper_2309_06973_amd.q8 import Q8, Q8Matrix

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2309_06973_amd", "csrc")

PROGRAM = r"""
#include <stdio.h>
#include <string.h>
#include "q8_plan.h"
using namespace shifter;
static int bad = 0;
static void want(const char* got, const char* part, int line) {
    if ((got == nullptr) != (part == nullptr) || (got && !strstr(got, part))) {
        printf("line %d: %s, expected %s\n", line, got ? got : "accepted", part ? part : "accepted");
        ++bad;
    }
}
#define WANT(expr, part) want(expr, part, __LINE__)
int main() {
    char* p = reinterpret_cast<char*>(0x1000);
    WANT(q8_bad_rows(p, 4, 3, 5, 5), nullptr);
    WANT(q8_bad_rows(p + 2, 2, 3, 5, 7), nullptr);
    WANT(q8_bad_rows(nullptr, 4, 0, 5, 5), nullptr);          // nothing to read
    WANT(q8_bad_rows(nullptr, 4, 3, 0, 0), nullptr);
    WANT(q8_bad_rows(nullptr, 4, 3, 5, 5), "NULL");
    WANT(q8_bad_rows(p + 2, 4, 3, 5, 5), "aligned");
    WANT(q8_bad_rows(p + 1, 2, 3, 5, 5), "aligned");
    WANT(q8_bad_rows(p, 4, 3, 5, 4), "smaller than a row");
    WANT(q8_bad_rows(p, 4, 1, 5, 0), nullptr);                // one row needs no stride
    WANT(q8_bad_rows(p, 4, 3, 5, (1ull << 32) + 1), "2^32");
    WANT(q8_bad_rows(p, 4, 1ull << 31, 5, 5), "rows or columns");
    WANT(q8_bad_rows(p, 4, 3, 1ull << 31, 1ull << 31), "rows or columns");
    WANT(q8_bad_rows(p, 4, ~0ull, ~0ull, ~0ull), "rows or columns");
    WANT(q8_bad_codes(p, p, 3, 17, 32), nullptr);
    WANT(q8_bad_codes(nullptr, nullptr, 0, 17, 0), nullptr);
    WANT(q8_bad_codes(nullptr, p, 3, 0, 0), nullptr);         // rows without columns have scales only
    WANT(q8_bad_codes(nullptr, p, 3, 17, 32), "NULL");
    WANT(q8_bad_codes(p, nullptr, 3, 17, 32), "NULL");
    WANT(q8_bad_codes(p, nullptr, 3, 0, 0), "NULL");
    WANT(q8_bad_codes(p + 8, p, 3, 17, 32), "16 bytes");
    WANT(q8_bad_codes(p, p, 3, 17, 40), "16 bytes");
    WANT(q8_bad_codes(p, p + 2, 3, 17, 32), "aligned");
    WANT(q8_bad_codes(p, p, 3, 17, 16), "smaller than a row");
    WANT(q8_bad_codes(p, p, 1, 17, 16), "smaller than a row");
    WANT(q8_bad_codes(p, p, 3, 17, (1u << 22) + 16), "2^22");
    WANT(q8_bad_codes(p, p, 1ull << 31, 17, 32), "rows or columns");
    WANT(q8_too_many(1u << 20, 1u << 14), nullptr);
    WANT(q8_too_many(1u << 20, 1u << 15), "more tiles");
    WANT(q8_too_many(0x7fffffff, 16), "more tiles");
    WANT(q8_too_many(1u << 27, 16), nullptr);
    WANT(q8_too_many(1, 1u << 26), "more tiles");
    WANT(q8_too_many(16, (1u << 26) - 16), nullptr);
    // workspace: the parts follow one another, every slice has rows, the rows are all in slices
    const uint64_t ms[] = {0, 1, 64, 127, 128, 129, 4095, 4096, 4097, 8191, 8192, 8193, 16384, 20000, 131071};
    const uint64_t ns[] = {1, 63, 500, 2048, 4097};
    int used[Q8_GRAD_KERNELS] = {0}, split = 0;
    for (uint64_t m : ms)
        for (uint64_t n : ns)
            for (uint64_t k : ns) {
                const Q8GradientPlan g = q8_gradient_plan(m, n, k);
                const bool is_small = m <= 16 || (m <= 2048 && n * k <= 1ull << 20 && m * n * k <= 1ull << 27);
                if ((g.kernel < 0) != is_small || (is_small && g.bytes != 0)) { printf("small %llu %llu %llu\n", (unsigned long long)m, (unsigned long long)n, (unsigned long long)k); ++bad; }
                if (is_small) continue;
                bool ok = m > 0 && g.ld >= m && g.ld < m + 128 && g.ld % 128 == 0 && g.slices <= Q8_SLICES && g.slice_rows % Q8_SLICE_ROWS == 0;
                ok = ok && (m <= Q8_WHOLE_ROWS ? g.slices == 0 : (uint64_t)g.slices * g.slice_rows >= m && (uint64_t)(g.slices - 1) * g.slice_rows < m);
                ok = ok && g.tops == 0 && g.slice_tops >= 4 * n && g.digits >= g.slice_tops + 4 * n * g.slices && g.digits % 256 == 0;
                ok = ok && g.kernel >= 0 && g.kernel < Q8_GRAD_KERNELS && g.parts >= 1 && g.parts <= Q8_PARTS && g.part_rows % 128 == 0;
                ok = ok && (uint64_t)g.parts * g.part_rows >= g.ld && (g.ld == 0 || (uint64_t)(g.parts - 1) * g.part_rows < g.ld);
                ok = ok && g.sums == g.codes + k * g.ld && g.sums % 128 == 0 && (m == 0 || g.bytes == g.sums + (g.parts > 1 ? 4 * g.parts * n * k : 0));
                if (ok) { ++used[g.kernel]; split += g.parts > 1; }
                ok = ok && g.codes >= g.digits + 3 * n * g.ld && g.codes % 128 == 0 && g.bytes >= (m ? g.codes + k * g.ld : 0);
                if (!ok) { printf("plan of %llu %llu %llu\n", (unsigned long long)m, (unsigned long long)n, (unsigned long long)k); ++bad; }
            }
    for (int q = 0; q < Q8_GRAD_KERNELS; ++q) if (!used[q]) { printf("gradient kernel %d is never taken\n", q); ++bad; }
    if (!split) { printf("rows are never split\n"); ++bad; }
    // kernels: few rows take the one without tiles, and every kernel is taken somewhere
    int taken[Q8_KERNELS] = {0};
    for (uint64_t m = 1; m <= 20000; m += 1 + m / 7)
        for (uint64_t n = 1; n <= 20000; n += 1 + n / 5)
            for (uint64_t k = 0; k <= Q8_MAX_K; k = k * 3 + 17) {
                const Q8Kernel q = q8_kernel_for(m, n, k);
                taken[q] += 1;
                const bool few = m <= Q8_FEW_ROWS || (m <= Q8_FEW_ROWS_MOST && n * k <= Q8_FEW_WEIGHTS);
                if (q >= Q8_KERNELS || (q == Q8_FEW) != few) { printf("kernel of %llu %llu %llu\n", (unsigned long long)m, (unsigned long long)n, (unsigned long long)k); ++bad; }
            }
    for (int q = 0; q < Q8_KERNELS; ++q) if (!taken[q]) { printf("kernel %d is never taken\n", q); ++bad; }
    if (q8_kernel_for(8192, 8192, 8192) != Q8_TILE_256x256 || q8_kernel_for(128, 4096, 4096) != Q8_TILE_64x64) { printf("ends\n"); ++bad; }
    printf("%d bad\n", bad);
    return bad != 0;
}
"""


def test_checks_and_plan(tmp_path):
    src = tmp_path / "q8.cpp"
    src.write_text(PROGRAM)
    exe = str(tmp_path / "q8")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


def test_layout_call_and_calls_without_a_context():
    assert S.shifter_weight_grad_q8_layout(0, 5, 5) == 0
    assert S.shifter_weight_grad_q8_layout(16, 5000, 7000) == S.shifter_weight_grad_q8_layout(60, 50, 70) == 0
    assert S.shifter_weight_grad_q8_layout(2100, 5, 7) >= 2176 * (3 * 5 + 7)
    with pytest.raises(S.ShifterError) as e:
        S.shifter_weight_grad_q8_layout(S.SHIFTER_Q8_MAX_SUM + 1, 5, 5)
    assert e.value.code == S.SHIFTER_ERR_CAPACITY
    with pytest.raises(S.ShifterError) as e:
        S.shifter_weight_grad_q8_layout(5, 1 << 31, 5)
    assert e.value.code == S.SHIFTER_ERR_INVALID_ARG
    lib = S.load_library()
    assert lib.shifter_weight_grad_q8_layout(1, 1, 1, None) == S.SHIFTER_ERR_INVALID_ARG
    assert lib.shifter_quantize_q8(None, None, 0, 0, 0, 0, 0, None, 0, None) == S.SHIFTER_ERR_INVALID_ARG
    assert lib.shifter_dequantize_q8(None, None, 0, None, 0, 0, None, 0, 0) == S.SHIFTER_ERR_INVALID_ARG
    assert lib.shifter_rms_norm_q8(None, None, 0, None, 0, 0, 0, 0, None, 0.0, None, 0, None, 0, None) == S.SHIFTER_ERR_INVALID_ARG
    assert lib.shifter_matmul_q8(None, None, 0, None, None, 0, None, 0, 0, 0, None, 0, None, 0, 0) == S.SHIFTER_ERR_INVALID_ARG
    assert lib.shifter_weight_grad_q8(None, None, 0, 0, None, 0, None, 0, 0, 0, None, 0, 0, None, 0, None, 0) == S.SHIFTER_ERR_INVALID_ARG


def test_matrix_refusals():
    z = lambda *shape: torch.zeros(*shape, dtype=torch.int8)
    m = Q8Matrix(z(3, 32), torch.zeros(3), 17)
    assert (m.rows, m.cols, m.ld) == (3, 17, 32)
    assert Q8Matrix(z(4, 64)[:, :32], torch.zeros(4), 20).ld == 64
    for q, s, c in ((z(3, 32).to(torch.uint8), torch.zeros(3), 17), (z(3, 32), torch.zeros(3).double(), 17),
                    (z(3, 32), torch.zeros(4), 17), (z(3, 32), torch.zeros(3), 33), (z(3, 32), torch.zeros(3), -1),
                    (z(32, 16).t(), torch.zeros(16), 17), (z(3, 2, 16), torch.zeros(3), 8),
                    (z(3, 32), torch.zeros(6)[::2], 17),
                    (z(1, 20), torch.zeros(1), 20), (z(84).as_strided((3, 20), (32, 1)), torch.zeros(3), 20)):
        with pytest.raises(ValueError):
            Q8Matrix(q, s, c)


def test_no_device_is_an_error():
    if torch.cuda.is_available():
        pytest.skip("a GPU is visible")
    with pytest.raises(RuntimeError):
        Q8()


def test_definition_of_codes():
    """Ties to even, both ends, zero rows and rows that are not finite."""
    q, a = Q.codes(np.array([[254.0, 127.0, 1.0, 3.0, -1.0, -3.0, 0.0, 5.0]]))       # 127 x / 254 = x / 2
    assert q.tolist() == [[127, 64, 0, 2, 0, -2, 0, 2]] and a[0] == 254.0            # 63.5 -> 64, .5 -> 0, 1.5 -> 2, 2.5 -> 2
    q, a = Q.codes(np.array([[0.0, -0.0], [1.0, np.inf], [np.nan, 1.0], [-2.0, 1e-40]]))
    assert q.tolist() == [[0, 0], [0, 0], [0, 0], [-127, 0]]
    assert a[0] == 0 and np.isnan(a[1]) and np.isnan(a[2]) and a[3] == 2.0
    q, s = Q.quantize(torch.tensor([[-5.0, 1.0, 0.5, -float("inf")]]), relu=True)
    assert q.tolist() == [[0, 127, 64, 0]] and s[0] == 1.0 / 127.0                   # 63.5 -> 64
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 40)).astype(np.float32).astype(np.float64)
    q, a = Q.codes(x)
    t = 127.0 * x / a[:, None]
    assert (np.abs(q - t) <= 0.5 + 1e-9).all()


def test_definition_of_the_gradient_against_differences():
    """dW of sum(g * (x W')) with x the values of an 8-bit matrix: central differences of the loss."""
    rng = np.random.default_rng(2)
    q = rng.integers(-127, 128, (6, 4)).astype(np.int8)
    s = rng.random(6).astype(np.float32)
    g = torch.from_numpy(rng.standard_normal((6, 3)).astype(np.float32))
    d, _ = Q.weight_grad(g, q, s)
    x = q.astype(np.float64) * s.astype(np.float64)[:, None]
    w = rng.standard_normal((3, 4))
    loss = lambda w_: float((Q.f64(g) * np.tanh(x @ w_.T * 0.01)).sum())
    # through a nonlinearity: its derivative joins g
    act = np.tanh(x @ w.T * 0.01)
    d, _ = Q.weight_grad(torch.from_numpy(Q.f64(g) * (1 - act ** 2) * 0.01), q, s)
    for i in range(3):
        for j in range(4):
            e = np.zeros_like(w)
            e[i, j] = 1e-5
            assert abs((loss(w + e) - loss(w - e)) / 2e-5 - d[i, j]) <= 1e-6 * max(1.0, abs(d[i, j]))
