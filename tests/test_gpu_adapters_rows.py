"""What a row of an adapters' call depends on: its own numbers and adapter, in calls of the same sizes."""
import pytest
import torch

from oracle import learn_oracle as L
from paper_2309_06973_amd.q8 import Q8, adapted
from test_gpu_adapters import DTYPES, near, rand, setup

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ops():
    o = Q8()
    yield o
    torch.cuda.synchronize()
    o.close()


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("m, n, k, rank, adapters", [(5, 300, 704, 16, 3), (40, 300, 700, 16, 9), (128, 200, 512, 8, 40), (300, 300, 700, 16, 5), (1000, 200, 333, 20, 12),
                                                     (2100, 130, 700, 16, 4), (9000, 70, 65, 16, 20), (200, 90, 700, 50, 6)])
def test_other_rows_do_not_matter(ops, m, n, k, rank, adapters, codes):
    """In calls of the same sizes a row is the same to the bit whatever the others hold, which adapters they have and whether these are finite."""
    for dtype in DTYPES:
        print(f"other rows m={m} n={n} k={k} rank={rank} adapters={adapters} {dtype} codes={codes}", flush=True)
        y, x, _, a, b, num, scale = setup(ops, m, n, k, rank, adapters, dtype, "random", codes)
        num[::3] = 1
        down = torch.empty(m, rank, device=DEV)
        out = ops.adapters(y, x, a, b, num, scale=scale, down=down)
        y2, x2, _, a2, b2, num2, _ = setup(ops, m, n, k, rank, adapters, dtype, "runs", codes, seed=77)
        num2 = torch.where(num2 == 1, 2, num2)
        a2[1], b2[1], num2[::3], y2[::3] = a[1], b[1], 1, y[::3]
        a2[0], b2[2] = NAN, INF
        if codes:
            x2.q[::3], x2.scale[::3] = x.q[::3], x.scale[::3]
        else:
            x2[::3] = x[::3]
        down2 = torch.empty(m, rank, device=DEV)
        again = ops.adapters(y2, x2, a2, b2, num2, scale=scale, down=down2)
        assert torch.equal(again[::3], out[::3]) and torch.equal(down2[::3], down[::3])


def test_the_same_every_time_in_the_adapters_order(ops):
    """Rows that are put in order first: where they land among their adapter's is not always the same, what they give is."""
    for m, adapters, codes in ((500, 8, False), (3000, 40, True), (9001, 12, False)):
        y, x, _, a, b, num, scale = setup(ops, m, 200, 264, 16, adapters, torch.bfloat16, "random", codes)
        g = rand(m, 200, dtype=torch.bfloat16, seed=4)
        every = lambda: (ops.adapters(y, x, a, b, num, scale=scale), *ops.adapters_grad(g, x, a, b, num, scale=scale))
        first = every()
        for _ in range(10):
            assert all(torch.equal(p, q) for p, q in zip(first, every()))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m, adapters", [(3, 2), (60, 20), (300, 3), (700, 20)])
def test_factors_below_the_normal_numbers(ops, m, adapters, dtype):
    """Activations and gradients that the type holds as its smallest numbers only, with adapters and scales that bring them back: none is taken for 0."""
    n, k, rank = 96, 160, 16
    y, _, _, a, b, num, scale = setup(ops, m, n, k, rank, adapters, dtype, "random")
    num[0] = 0
    least, up, by = (2.0 ** -24, 1.0, 2.0 ** 14) if dtype == torch.float16 else (2.0 ** -133, 2.0 ** 20, 2.0 ** 100)
    some = lambda cols, seed: (torch.randint(-100, 101, (m, cols), generator=torch.Generator().manual_seed(seed)) * least).to(dtype).to(DEV)
    x, g, a, b, scale = some(k, 1), some(n, 2), a * up, b * up, scale * by
    y = torch.zeros(m, n, device=DEV)
    ref = L.Adapters(y, x, a, b, num, scale)
    down = torch.empty(m, rank, device=DEV)
    out = ops.adapters(y, x, a, b, num, scale=scale, down=down)
    near(down, ref.down, ref.off_down, torch.float32, "down")
    near(out, ref.out, ref.off, torch.float32, "out")
    for name, got, t in zip(("dx", "da", "db"), ops.adapters_grad(g, x, a, b, num, scale=scale, down=down), (dtype, torch.float32, torch.float32)):
        near(got, *ref.grads(g)[name], t, name)


@pytest.mark.parametrize("default", [torch.float64, torch.bfloat16])
def test_adapted_whatever_torch_makes_by_default(ops, default):
    y, x, _, a, b, num, scale = setup(ops, 24, 50, 40, 8, 3, torch.float32, "random")
    g = rand(24, 50, dtype=torch.float32, seed=8)
    ref = L.Adapters(y, x, a, b, num, scale)
    leaf = a.clone().requires_grad_()
    was = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        out = adapted(y, x, leaf, b, num, ops, scale=scale)
        (da,) = torch.autograd.grad(out, leaf, g)
    finally:
        torch.set_default_dtype(was)
    near(out, ref.out, ref.off, torch.float32, "out")
    near(da, *ref.grads(g)["da"], torch.float32, "da")
