"""Low-rank adapters of many requests and their gradients against the definition in 64 bits; how far they may be off is
derived in oracle.learn_oracle."""
import numpy as np
import pytest
import torch

from oracle import learn_oracle as L
from paper_2309_06973_amd import shifter as S
from paper_2309_06973_amd.q8 import Q8, Q8Matrix, adapted

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ops():
    o = Q8()
    yield o
    torch.cuda.synchronize()
    o.close()


def rand(*shape, dtype, seed, size=1.0, gap=0, shift=0):
    g = torch.Generator().manual_seed(seed)
    if len(shape) == 2:
        rows, cols = shape
        x = (size * torch.randn(rows * (cols + gap) + shift, generator=g)).to(dtype).to(DEV)
        return x[shift:].view(rows, cols + gap)[:, :cols]
    return (size * torch.randn(*shape, generator=g)).to(dtype).to(DEV)


def numbers(m, adapters, pattern, seed):
    g = torch.Generator().manual_seed(seed)
    if pattern == "one":
        return torch.full((m,), adapters - 1).to(DEV)
    if pattern == "random":
        return torch.randint(-1, adapters, (m,), generator=g).to(DEV)
    if pattern == "none":
        return torch.full((m,), -7).to(DEV)
    at = torch.sort(torch.randint(0, m + 1, (adapters - 1,), generator=g)).values          # runs, some empty
    return torch.randperm(adapters, generator=g)[torch.bucketize(torch.arange(m), at, right=True)].to(DEV)


def near(got, want, off, dtype, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, what
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    ok = torch.isfinite(want)
    bound = (off + L.HALF_STEP[dtype] * (want.abs() + off) + L.LEAST[dtype])[ok]
    bad = (got[ok] - want[ok]).abs() > bound
    assert not bad.any(), (what, got[ok][bad][:3], want[ok][bad][:3], bound[bad][:3])


def setup(ops, m, n, k, rank, adapters, dtype, pattern, codes=False, y_dtype=None, gap=0, shift=0, seed=1):
    x = rand(m, k, dtype=dtype, seed=seed, gap=gap, shift=shift)
    values = x
    if codes:
        x = ops.quantize(x)
        values = x.q[:, :k].double() * x.scale.double()[:, None]
    a = rand(adapters, rank, k, dtype=dtype, seed=seed + 1, size=max(k, 1) ** -0.5)
    b = rand(adapters, n, rank, dtype=dtype, seed=seed + 2, size=rank ** -0.5)
    y = rand(m, n, dtype=y_dtype or dtype, seed=seed + 3, gap=gap, shift=shift)
    which = numbers(m, adapters, pattern, seed + 4)
    scale = (0.5 + torch.rand(adapters, generator=torch.Generator().manual_seed(seed))).to(DEV)
    return y, x, values, a, b, which, scale


SIZES = [(1, 1, 1, 1, 1), (1, 64, 64, 16, 3), (2, 65, 63, 3, 2), (3, 7, 5, 4, 1), (5, 300, 8, 8, 4), (16, 64, 9, 12, 5), (17, 255, 200, 16, 17), (33, 257, 127, 17, 3),
         (48, 100, 321, 32, 32), (64, 17, 129, 48, 4), (100, 1000, 64, 64, 2), (31, 129, 777, 65, 3), (40, 70, 130, 100, 6), (9, 1, 2000, 128, 2), (256, 130, 65, 5, 7),
         (257, 130, 65, 5, 7), (300, 90, 1000, 20, 3), (700, 513, 40, 33, 70), (1025, 64, 192, 16, 5), (7, 5000, 4096, 16, 3)]


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("which", range(len(SIZES)))
def test_adapters(ops, which, dtype, codes):
    m, n, k, rank, adapters = SIZES[which]
    for pattern, y_dtype, gap, shift in (("runs", dtype, 0, 0), ("random", torch.float32, 3, 1), ("one", torch.bfloat16, 0, 5), ("none", torch.float16, 8, 0)):
        print(f"adapters m={m} n={n} k={k} rank={rank} adapters={adapters} {dtype} codes={codes} {pattern} y={y_dtype} gap={gap}", flush=True)
        y, x, values, a, b, num, scale = setup(ops, m, n, k, rank, adapters, dtype, pattern, codes, y_dtype, gap, shift)
        ref = L.Adapters(y, values, a, b, num, scale)
        out = ops.adapters(y, x, a, b, num, scale=scale)
        near(out, ref.out, ref.off, y_dtype, "out")
        assert torch.equal(out[num < 0], y[num < 0])
        down = torch.full((m, rank), 9.0, device=DEV)
        wide = torch.full((m, n + 5), 7.0, dtype=y_dtype, device=DEV)
        assert torch.equal(ops.adapters(y, x, a, b, num, scale=scale, out=wide[:, 2:n + 2], down=down), out)
        assert (wide[:, :2] == 7).all() and (wide[:, n + 2:] == 7).all()
        near(down, ref.down, ref.off_down, torch.float32, "down")
        z = y.clone()
        assert ops.adapters(z, x, a, b, num, scale=scale, out=z) is z and torch.equal(z, out)
        if pattern == "runs":
            plain = L.Adapters(y, values, a, b, num)
            near(ops.adapters(y, x, a, b, num), plain.out, plain.off, y_dtype, "out without scales")


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, n, k, rank, adapters", [(1, 4096, 4096, 16, 8), (1, 4097, 4104, 16, 8), (1, 17000, 64, 31, 2), (3, 1000, 3880, 16, 1), (8, 63, 3000, 32, 9), (16, 300, 1024, 1, 40),
                                                    (17, 1025, 8, 12, 3), (48, 2500, 1088, 16, 32), (128, 5000, 1000, 20, 40), (129, 300, 1000, 20, 40), (100, 70, 0, 8, 5)])
def test_few_rows_of_small_adapters(ops, m, n, k, rank, adapters, dtype, codes):
    """Around what one launch does for, columns that end anywhere, rows that name no adapter among others."""
    for pattern, gap, shift in (("random", 0, 0), ("runs", 8, 3), ("one", 4, 0)):
        print(f"few rows m={m} n={n} k={k} rank={rank} adapters={adapters} {dtype} codes={codes} {pattern} gap={gap}", flush=True)
        y, x, values, a, b, num, scale = setup(ops, m, n, k, rank, adapters, dtype, pattern, codes, torch.bfloat16, gap, shift)
        if m > 2:
            num[1], num[2] = -1, adapters
        ref = L.Adapters(y, values, a, b, num, scale)
        down = torch.full((m, rank), 9.0, device=DEV)
        out = ops.adapters(y, x, a, b, num, scale=scale, down=down)
        near(out, ref.out, ref.off, torch.bfloat16, "out")
        near(down, ref.down, ref.off_down, torch.float32, "down")
        z = y.clone()
        ops.adapters(z, x, a, b, num, scale=scale, out=z)
        assert torch.equal(torch.nan_to_num(z), torch.nan_to_num(out))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, n, rank", [(1, 64, 3), (5, 2048, 16), (100, 1000, 8), (128, 4096, 4), (16, 300, 40), (300, 512, 16)])
def test_x_is_y_in_place(ops, m, n, rank, dtype):
    x, _, _, a, b, num, scale = setup(ops, m, n, n, rank, 5, dtype, "random")
    num = num.clamp(min=0)
    want = ops.adapters(x, x, a, b, num, scale=scale)
    ref = L.Adapters(x, x, a, b, num, scale)
    near(want, ref.out, ref.off, dtype, "out")
    for _ in range(5):
        z = x.clone()
        ops.adapters(z, z, a, b, num, scale=scale, out=z)
        near(z, ref.out, ref.off, dtype, "in place")


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("which", range(len(SIZES)))
def test_gradients(ops, which, dtype, codes):
    m, n, k, rank, adapters = SIZES[which]
    for pattern, gap, shift in (("runs", 0, 0), ("random", 3, 1), ("none", 0, 0)):
        print(f"adapters_grad m={m} n={n} k={k} rank={rank} adapters={adapters} {dtype} codes={codes} {pattern} gap={gap}", flush=True)
        y, x, values, a, b, num, scale = setup(ops, m, n, k, rank, adapters, dtype, pattern, codes, dtype, gap, shift)
        g = rand(m, n, dtype=dtype, seed=9, gap=gap, shift=shift)
        ref = L.Adapters(y, values, a, b, num, scale)
        down = torch.empty(m, rank, device=DEV)
        ops.adapters(y, x, a, b, num, scale=scale, down=down)
        for kept in (down, None):
            dx, da, db = ops.adapters_grad(g, x, a, b, num, scale=scale, down=kept)
            for name, got, t in (("dx", dx, dtype), ("da", da, torch.float32), ("db", db, torch.float32)):
                near(got, *ref.grads(g)[name], t, name)
            assert (dx[num < 0] == 0).all()
        none, da2, db2 = ops.adapters_grad(g, x, a, b, num, scale=scale, dx=False)
        assert none is None and torch.equal(da, da2) and torch.equal(db, db2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, n, k, rank, adapters", [(257, 70, 64, 16, 8), (600, 200, 150, 16, 9), (3000, 130, 70, 20, 40), (2048, 64, 65, 32, 300), (9001, 65, 40, 8, 12),
                                                    (700, 300, 33, 50, 4094), (700, 300, 33, 12, 4095)])
def test_rows_in_the_order_of_their_adapters(ops, m, n, k, rank, adapters, dtype):
    """More rows than a wavefront's tiles for each of many adapters, forward and back; more rows than the order's block holds."""
    for pattern, codes in (("random", False), ("runs", True), ("one", False), ("none", False)):
        print(f"in order m={m} n={n} k={k} rank={rank} adapters={adapters} {dtype} codes={codes} {pattern}", flush=True)
        y, x, values, a, b, num, scale = setup(ops, m, n, k, rank, adapters, dtype, pattern, codes)
        num[3] = adapters                    # names none
        ref = L.Adapters(y, values, a, b, num, scale)
        down = torch.full((m, rank), 9.0, device=DEV)
        out = ops.adapters(y, x, a, b, num, scale=scale, down=down)
        near(out, ref.out, ref.off, dtype, "out")
        near(down, ref.down, ref.off_down, torch.float32, "down")
        z = y.clone()
        assert torch.equal(ops.adapters(z, x, a, b, num, scale=scale, out=z)[num < adapters], out[num < adapters])
        g = rand(m, n, dtype=dtype, seed=9)
        for kept in (down, None):
            for name, got, t in zip(("dx", "da", "db"), ops.adapters_grad(g, x, a, b, num, scale=scale, down=kept), (dtype, torch.float32, torch.float32)):
                near(got, *ref.grads(g)[name], t, name)


def test_no_rows_and_no_columns(ops):
    for m, n, k, adapters in ((0, 5, 7, 2), (3, 0, 7, 2), (3, 5, 0, 2), (3, 5, 7, 0), (0, 0, 0, 0)):
        y, x, a, b = torch.ones(m, n, device=DEV), torch.ones(m, k, device=DEV), torch.ones(adapters, 4, k, device=DEV), torch.ones(adapters, n, 4, device=DEV)
        num = torch.tensor([0, -1, 9][:m], dtype=torch.int64, device=DEV)
        ref = L.Adapters(y, x, a, b, num)
        down = torch.full((m, 4), 5.0, device=DEV)
        near(ops.adapters(y, x, a, b, num, down=down), ref.out, ref.off, torch.float32, "out")
        near(down, ref.down, ref.off_down, torch.float32, "down")
        for name, got in zip(("dx", "da", "db"), ops.adapters_grad(torch.ones(m, n, device=DEV), x, a, b, num)):
            near(got, *ref.grads(torch.ones(m, n))[name], torch.float32, name)


@pytest.mark.parametrize("m", [40, 400])
def test_nothing_reaches_another_row(ops, m):
    """An adapter that is not finite, a row that is not, numbers that name no adapter: their own rows alone."""
    y, x, _, a, b, num, _ = setup(ops, m, 200, 150, 20, 6, torch.float32, "random")
    num[5] = 6
    num[6] = 1 << 40
    num[7] = -(1 << 60)
    num[8] = 1
    clean = ops.adapters(y, x, a, b, num)
    a[2], b[4, 3] = NAN, INF
    x[8] = NAN
    got = ops.adapters(y, x, a, b, num)
    bad = (num == 2) | (num == 4) | (num >= 6)
    bad[8] = True
    assert torch.equal(got[~bad], clean[~bad]) and torch.isnan(got[(num == 2) | (num >= 6)]).all() and torch.equal(got[7], y[7])
    assert torch.isnan(got[8]).all() and not torch.isfinite(got[num == 4][:, 3]).any()
    g = rand(m, 200, dtype=torch.float32, seed=3)
    dx, da, db = ops.adapters_grad(g, x, a, b, num)
    fine = [i for i in range(6) if i not in (1, 2, 4)]
    assert torch.isfinite(da[fine]).all() and torch.isfinite(db[fine]).all() and torch.isnan(da[1]).any()
    assert torch.isfinite(dx[~bad]).all() and torch.isnan(dx[num >= 6]).all() and (dx[7] == 0).all()
    first = ops.adapters(y, x, a, b, num)
    assert torch.equal(first[num >= 0].isnan(), got[num >= 0].isnan())


@pytest.mark.parametrize("m", [50, 1000])
def test_a_rows_neighbours_do_not_matter(ops, m):
    """A row's result is the same to the bit whatever order the rows of its call come in."""
    for dtype in DTYPES:
        y, x, _, a, b, num, scale = setup(ops, m, 300, 700, 16, 9, dtype, "random")
        out = ops.adapters(y, x, a, b, num, scale=scale)
        order = torch.randperm(m, generator=torch.Generator().manual_seed(2)).to(DEV)
        assert torch.equal(ops.adapters(y[order], x[order], a, b, num[order], scale=scale), out[order])


def test_the_same_every_time(ops):
    y, x, _, a, b, num, scale = setup(ops, 2000, 600, 800, 16, 3, torch.bfloat16, "runs")
    g = rand(2000, 600, dtype=torch.bfloat16, seed=4)
    first = (ops.adapters(y, x, a, b, num, scale=scale), *ops.adapters_grad(g, x, a, b, num, scale=scale))
    for _ in range(10):
        again = (ops.adapters(y, x, a, b, num, scale=scale), *ops.adapters_grad(g, x, a, b, num, scale=scale))
        assert all(torch.equal(p, q) for p, q in zip(first, again))


def test_large(ops):
    """Prompts of several requests in the shape of a wide layer, all of it against 64 bits on a sample of rows and columns."""
    m, n, k, rank, many = 8192, 4096, 4096, 16, 6
    y, x, values, a, b, num, scale = setup(ops, m, n, k, rank, many, torch.bfloat16, "runs")
    out = ops.adapters(y, x, a, b, num, scale=scale)
    rows, cols = torch.arange(0, m, 61, device=DEV), torch.arange(0, n, 37, device=DEV)
    ref = L.Adapters(y[rows][:, cols], x[rows], a, b[:, cols], num[rows], scale)
    near(out[rows][:, cols], ref.out, ref.off, torch.bfloat16, "out")
    g = rand(m, n, dtype=torch.bfloat16, seed=5)
    dx, da, db = ops.adapters_grad(g, x, a, b, num, scale=scale)
    some = torch.arange(0, n, 97, device=DEV)
    ref = L.Adapters(y, x, a, b, num, scale)
    want = ref.grads(g)
    near(dx[rows], want["dx"][0][rows.cpu()], want["dx"][1][rows.cpu()], torch.bfloat16, "dx")
    near(da[:, :, some], want["da"][0][:, :, some.cpu()], want["da"][1][:, :, some.cpu()], torch.float32, "da")
    near(db[:, some], want["db"][0][:, some.cpu()], want["db"][1][:, some.cpu()], torch.float32, "db")


def test_offsets_beyond_32_bits(ops):
    """Rows of x and y that start 2^32 elements in, and an adapter behind 2^31 others' elements."""
    ld = (1 << 32) - 16
    buf = torch.zeros(ld + 300, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(buf, (2, 128), (ld, 1))
    y = torch.as_strided(buf, (2, 100), (ld, 1), 136)
    x.copy_(rand(2, 128, dtype=torch.bfloat16, seed=1))
    y.copy_(rand(2, 100, dtype=torch.bfloat16, seed=2))
    many = (1 << 31) // (128 * 16) + 2
    a = torch.zeros(many, 16, 128, dtype=torch.bfloat16, device=DEV)
    b = torch.zeros(many, 100, 16, dtype=torch.bfloat16, device=DEV)
    a[-1], b[-1] = rand(16, 128, dtype=torch.bfloat16, seed=3), rand(100, 16, dtype=torch.bfloat16, seed=4)
    num = torch.tensor([-1, many - 1], device=DEV)
    small = L.Adapters(y, x, a[-1:], b[-1:], torch.tensor([-1, 0]))
    ops.adapters(y, x, a, b, num, out=y)
    near(y, small.out, small.off, torch.bfloat16, "out")


@pytest.mark.parametrize("codes", [False, True])
def test_autograd(ops, codes):
    """Through torch's graph against the formula's gradients, and against differences."""
    y, x, values, a, b, num, scale = setup(ops, 24, 50, 40, 8, 3, torch.float32, "random", codes)
    y, a, b = (t.clone().requires_grad_() for t in (y, a, b))
    if not codes:
        x = x.clone().view(4, 6, 40).requires_grad_()
    out = adapted(y.view(4, 6, 50), x, a, b, num.view(4, 6), ops, scale=scale)
    g = rand(24, 50, dtype=torch.float32, seed=8)
    out.backward(g.view(4, 6, 50))
    ref = L.Adapters(y, values, a, b, num, scale)
    want = ref.grads(g)
    assert torch.equal(y.grad, g)
    near(a.grad, *want["da"], torch.float32, "da")
    near(b.grad, *want["db"], torch.float32, "db")
    if not codes:
        near(x.grad.view(24, 40), *want["dx"], torch.float32, "dx")
    loss = lambda a_, b_: float((L.Adapters(y, values, a_, b_, num, scale).out * g.cpu().double()).sum())
    for t, other, at in ((a, b, (1, 3, 7)), (b, a, (2, 11, 5))):
        f = []
        for step in (0.5, -0.5):                # linear in each: differences are exact
            v = t.detach().double().clone()
            v[at] += step
            f.append(loss(v, other) if t is a else loss(other, v))
        assert abs(f[0] - f[1] - float(t.grad[at])) < 1e-4


def test_second_derivative_and_lost_gradients(ops):
    y, x, _, a, b, num, scale = setup(ops, 24, 50, 40, 8, 3, torch.float32, "random")
    leaf = a.clone().requires_grad_()
    out = adapted(y, x, leaf, b, num, ops)
    (da,) = torch.autograd.grad(out.sum(), leaf, create_graph=True)
    with pytest.raises(RuntimeError, match="no derivative"):
        da.square().sum().backward()
    with pytest.raises(RuntimeError, match="passes no gradients on"):
        ops.adapters(y, x, leaf, b, num).sum().backward()
    with pytest.raises(ValueError, match="needs a gradient"):
        ops.adapters(y, x, leaf, b, num, out=y)
    with pytest.raises(RuntimeError, match="passes no gradients on"):
        ops.adapters_grad(y, x, leaf, b, num)[2].sum().backward()
    with pytest.raises(ValueError, match="scale needs a gradient"):
        adapted(y, x, a, b, num, ops, scale=scale.clone().requires_grad_())
    with pytest.raises(ValueError, match="y must have"):
        adapted(y.bfloat16(), x, a, b, num, ops)
    with pytest.raises(ValueError, match="which must have"):
        adapted(y, x, a, b, num[:3], ops)


@pytest.mark.parametrize("many", [5, 20])
def test_recorded(ops, many):
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        own = Q8()
        y, x, _, a, b, num, scale = setup(own, 300, 500, 700, 16, many, torch.bfloat16, "random")
        g = rand(300, 500, dtype=torch.bfloat16, seed=5)
        down = torch.empty(300, 16, device=DEV)
        own.adapters_grad(g, x, a, b, num)
        torch.cuda.synchronize()
        graphs = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                out = own.adapters(y, x, a, b, num, scale=scale, down=down)
                grads = own.adapters_grad(g, x, a, b, num, scale=scale, down=down)
            graphs.append((graph, (out, *grads)))
        for i in range(4):
            x.copy_(rand(300, 700, dtype=torch.bfloat16, seed=30 + i))
            num.copy_(numbers(300, many, "random", 40 + i))
            for graph, got in graphs:
                for t in got:
                    t.fill_(3.0)
                graph.replay()
                want = (own.adapters(y, x, a, b, num, scale=scale), *own.adapters_grad(g, x, a, b, num, scale=scale))
                torch.cuda.synchronize()
                assert all(torch.equal(p, q) for p, q in zip(got, want))
        leaf = a.clone().requires_grad_()
        with pytest.raises(RuntimeError, match="can not be recorded"):
            with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=stream):
                adapted(y, x, leaf, b, num, own)
        torch.cuda.synchronize()
        own.close()


def test_refusals(ops):
    y, x, _, a, b, num, scale = setup(ops, 4, 50, 40, 8, 3, torch.float32, "random")
    ok = dict(y=y, x=x, a=a, b=b, which=num)
    wide = torch.zeros(4, 60, device=DEV)
    for change, what in ((dict(x=x.bfloat16()), "a's type"), (dict(x=x[:, :39]), "a's columns"), (dict(y=y[:3]), "y must have"), (dict(a=a.double()), "a must be"),
                         (dict(a=a[0]), "a must be"), (dict(a=a.transpose(1, 2)), "a must be"), (dict(b=b.half()), "b must be"), (dict(b=b[:2]), "b must be"),
                         (dict(b=b[:, :, :4]), "b must be"), (dict(which=num.int()), "int64"), (dict(which=num[:3]), "int64"), (dict(scale=scale[:2]), "scale"),
                         (dict(out=y.bfloat16()), "out must have"), (dict(out=wide), "out must have"), (dict(down=torch.zeros(4, 9, device=DEV)), "down must have"),
                         (dict(down=torch.zeros(4, 8, dtype=torch.float16, device=DEV)), "down must have"), (dict(x=None), "Q8Matrix"), (dict(which=num.cpu()), "not on"),
                         (dict(x=ops.quantize(x[:, :32].contiguous())), "a's columns")):
        with pytest.raises(ValueError, match=what):
            ops.adapters(**{**ok, **change})
    with pytest.raises(S.ShifterError, match="1 to 128"):
        ops.adapters(y, x, torch.zeros(1, 129, 40, device=DEV), torch.zeros(1, 50, 129, device=DEV), num)
    with pytest.raises(S.ShifterError, match="1 to 128"):
        ops.adapters(y, x, torch.zeros(1, 0, 40, device=DEV), torch.zeros(1, 50, 0, device=DEV), num)
    with pytest.raises(ValueError, match="g must have"):
        ops.adapters_grad(y.bfloat16(), x, a, b, num)
    with pytest.raises(S.ShifterError) as e:
        S.shifter_adapters_layout((1 << 25) + 1, 1, 1, 1, 1)
    assert e.value.code == S.SHIFTER_ERR_CAPACITY
    with pytest.raises(S.ShifterError, match="more columns of all adapters") as e:
        S.shifter_adapters_grad_layout(1, 1 << 20, 1 << 20, 1, 1 << 10, 0)
    assert e.value.code == S.SHIFTER_ERR_CAPACITY
    need = S.shifter_adapters_layout(4, 50, 40, 8, 3)
    work = torch.zeros(need, dtype=torch.uint8, device=DEV)
    fine = dict(d_x=x, ld_x=40, m=4, n=50, k=40, rank=8, adapters=3, d_a=a, d_b=b, d_which=num, d_y=y, ld_y=50, d_out=y, ld_out=50, d_work=work, work_bytes=need)
    for change, what in ((dict(work_bytes=need - 1), "too small"), (dict(d_work=work.data_ptr() + 16), "256-byte"), (dict(d_which=None), "NULL"), (dict(d_a=None), "NULL"),
                         (dict(dtype=9), "element type"), (dict(y_dtype=9), "element type"), (dict(ld_out=51), "another stride"), (dict(ld_x=39), "stride"),
                         (dict(d_out=None), "NULL"), (dict(d_a=a.data_ptr() + 1), "aligned")):
        with pytest.raises(S.ShifterError, match=what):
            S.shifter_adapters(ops.ctx, **{**fine, **change})
    need = S.shifter_adapters_grad_layout(4, 50, 40, 8, 3, 0)
    work, da, db, dx = torch.zeros(need, dtype=torch.uint8, device=DEV), torch.zeros_like(a), torch.zeros_like(b), torch.zeros_like(x)
    fine = dict(d_x=x, ld_x=40, m=4, n=50, k=40, rank=8, adapters=3, d_a=a, d_b=b, d_which=num, d_g=y, ld_g=50, d_dx=dx, ld_dx=40, d_da=da, d_db=db, d_work=work,
                work_bytes=need)
    for change, what in ((dict(work_bytes=need - 1), "too small"), (dict(d_da=None), "NULL"), (dict(d_dx=x), "read to the end"), (dict(d_g=None), "NULL")):
        with pytest.raises(S.ShifterError, match=what):
            S.shifter_adapters_grad(ops.ctx, **{**fine, **change})
    S.shifter_adapters_grad(ops.ctx, **fine)
    torch.cuda.synchronize()
