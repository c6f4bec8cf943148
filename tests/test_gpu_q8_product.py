"""The 8-bit integer product and the weight gradient against their definition in 64 bits, and
both inside a recorded graph and behind autograd.

Product: the sum of whole numbers is exact; its conversion, the two scales and the bias' sum round
once each (the scale of the column and the bias in one step): at most 3.1 half steps of the
product's magnitude and one of the result in fp32, then half a step of the element type.
Gradient: the bound that the interface states, worked out per entry by the definition's side, and
one fp32 rounding of what it is added to."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as Q
from paper_2309_06973_amd import shifter as S
from paper_2309_06973_amd.q8 import Q8, Q8Matrix, checkpointed_linear

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ops():
    o = Q8()
    yield o
    torch.cuda.synchronize()
    o.close()


def matrix(rows, cols, seed, extra=0, fill=-128, ends=False):
    """(8-bit matrix with other bytes behind its columns, codes, scales)."""
    rng = np.random.default_rng(seed)
    q = rng.choice([-128, 127], (rows, cols)) if ends else rng.integers(-128, 128, (rows, cols))
    s = np.exp(rng.standard_normal(rows)).astype(np.float32) * 0.01
    ld = -(-cols // 16) * 16 + extra
    buf = torch.full((rows, ld), fill, dtype=torch.int8, device=DEV)
    buf[:, :cols] = torch.from_numpy(q.astype(np.int8)).to(DEV)
    return Q8Matrix(buf, torch.from_numpy(s).to(DEV), cols), q.astype(np.int8), s


def check_product(ops, m, n, k, dtype, seed=0, bias=False, relu=False, gap=0, ends=False, extra=0):
    print(f"product m={m} n={n} k={k} {dtype} bias={bias} relu={relu} gap={gap}", flush=True)
    a, qa, sa = matrix(m, k, seed, extra, ends=ends)
    b, qb, sb = matrix(n, k, seed + 1, 2 * extra, fill=127, ends=ends)
    bv = np.random.default_rng(seed + 2).standard_normal(n).astype(np.float32) if bias else None
    out = torch.full((m, n + gap), 3.0, dtype=Q.DTYPES[dtype], device=DEV)
    ops.matmul(a, b, bias=torch.from_numpy(bv).to(DEV) if bias else None, relu=relu, out=out[:, :n])
    want, mag = Q.product(qa, sa, qb, sb, bv, relu)
    got = Q.f64(out[:, :n])
    assert (np.abs(got - want) <= 3.1 * Q.U32 * mag + (Q.HALF_STEP[dtype] + 1.01 * Q.U32) * np.abs(want)
            + 1.01 * Q.LEAST[dtype] + Q.TINY32).all()
    assert (out[:, n:] == 3.0).all()


EDGES = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200, 255, 257]


@pytest.mark.parametrize("m", EDGES)
def test_product_rows(ops, m):
    check_product(ops, m, 65, 130, "fp32", seed=m)
    check_product(ops, m, 300, 77, "bf16", seed=m, bias=True, gap=1)


@pytest.mark.parametrize("n", EDGES)
def test_product_columns(ops, n):
    check_product(ops, 3, n, 200, "bf16", seed=n)
    check_product(ops, 140, n, 200, "fp16", seed=n, relu=True, gap=3)


@pytest.mark.parametrize("k", [0, 1, 3, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 500, 1000, 4100])
def test_product_sums(ops, k):
    for m in (1, 7, 20, 50, 100, 270):
        check_product(ops, m, 70, k, "fp32", seed=k + m, bias=True, extra=16 * (m % 3))


@pytest.mark.parametrize("m,n,k", [(1, 4096, 1000), (16, 2049, 640), (40, 515, 3000), (64, 1000, 999), (130, 1000, 999),
                                   (300, 4000, 70), (1000, 1100, 300), (2100, 2300, 260), (5000, 20, 100), (3, 40000, 48),
                                   (4000, 2047, 500), (4090, 4001, 1003)])
def test_product_sizes(ops, m, n, k):
    for dtype in Q.DTYPES:
        check_product(ops, m, n, k, dtype, seed=m, bias=True, relu=dtype == "fp16")


@pytest.mark.parametrize("m", [1, 30, 90, 300])
def test_product_longest_sums(ops, m):
    """131071 products of codes at both ends: the sums reach 2^31 - 2^14."""
    k = S.SHIFTER_Q8_MAX_SUM
    a = torch.full((m, k + 1), -128, dtype=torch.int8, device=DEV)
    b = torch.full((33, k + 1), -128, dtype=torch.int8, device=DEV)
    b[1] = 127
    one = lambda n: torch.ones(n, device=DEV)
    c = ops.matmul(Q8Matrix(a, one(m), k), Q8Matrix(b, one(33), k), dtype=torch.float32)
    assert (c[:, 0] == float(np.float32(128 * 128 * k))).all() and (c[:, 1] == float(np.float32(-128 * 127 * k))).all()
    check_product(ops, m, 5, k, "fp32", ends=True)
    with pytest.raises(S.ShifterError) as e:
        S.shifter_matmul_q8(ops.ctx, a, k + 1, one(m), b, k + 1, one(33), m, 33, k + 1, None, 0, c, 0, 33)
    assert e.value.code == S.SHIFTER_ERR_CAPACITY


def test_product_scales(ops):
    """A NaN scale makes its row or column NaN (through ReLU too), zero scales give the bias, scales
    whose product leaves the numbers' range do not."""
    for m in (5, 40, 200):
        a, qa, sa = matrix(m, 40, 1)
        b, qb, sb = matrix(90, 40, 2)
        a.scale[2] = float("nan")
        a.scale[3] = 0.0
        b.scale[7] = float("nan")
        a.scale[4], b.scale[8] = 1e-30, 1e-30
        a.scale[1], b.scale[9] = 1e25, 1e-36
        bias = torch.randn(90, device=DEV)
        c = ops.matmul(a, b, bias=bias, relu=True, dtype=torch.float32)
        assert torch.isnan(c[2]).all() and torch.isnan(c[:, 7]).all() and int(torch.isnan(c).sum()) == m + 90 - 1
        ok = torch.arange(90, device=DEV) != 7
        assert torch.equal(c[3][ok], bias[ok].clamp(min=0))
        assert torch.equal(c[4, 8], bias[8].clamp(min=0))
        want, mag = Q.product(qa[1:2], np.array([1e25], dtype=np.float32), qb[9:10], np.array([1e-36], dtype=np.float32))
        c = ops.matmul(a, b, dtype=torch.float32)
        assert abs(float(c[1, 9]) - want[0, 0]) <= 4 * Q.U32 * mag[0, 0] + 40 * 2.0 ** -126
    z = Q8Matrix(torch.zeros((0, 48), dtype=torch.int8, device=DEV), torch.zeros(0, device=DEV), 40)
    assert ops.matmul(z, b).shape == (0, 90) and ops.matmul(b, z).shape == (90, 0)


def test_product_far_offsets(ops):
    """Codes of both operands and results more than 2^32 bytes from the first."""
    rows, ld, k = 1100, 1 << 22, 100
    buf = torch.empty((rows, ld), dtype=torch.int8, device=DEV)
    small, q, s = matrix(rows, k, 3)
    buf[:, :k] = small.q[:, :k]
    far = Q8Matrix(buf, small.scale, k)
    b, qb, sb = matrix(70, k, 4)
    want = ops.matmul(small, b, dtype=torch.float32)
    assert torch.equal(ops.matmul(far, b, dtype=torch.float32), want)
    assert torch.equal(ops.matmul(b, far, dtype=torch.float32), ops.matmul(b, small, dtype=torch.float32))
    c = torch.empty((rows, 1 << 20), dtype=torch.float32, device=DEV)[:, :70]
    ops.matmul(small, b, out=c)
    assert torch.equal(c, want)
    exact, mag = Q.product(q, s, qb, sb)
    assert (np.abs(Q.f64(want) - exact) <= 4.2 * Q.U32 * mag + Q.TINY32).all()


# ---- the weight gradient ------------------------------------------------------------------

def grads(m, n, dtype, seed, gap=0, shift=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m * (n + gap) + shift, generator=g) * torch.exp(torch.randn(m * (n + gap) + shift, generator=g)) * 1e-3
    return x.to(Q.DTYPES[dtype]).to(DEV)[shift:].view(m, n + gap)[:, :n]


def check_gradient(ops, m, n, k, dtype, seed=0, mask=False, accumulate=False, gap=0, shift=0, g=None, ends=False):
    print(f"gradient m={m} n={n} k={k} {dtype} mask={mask} accumulate={accumulate} gap={gap}", flush=True)
    x, q, s = matrix(m, k, seed, extra=16 * (gap % 3), ends=ends)
    g = grads(m, n, dtype, seed, gap, shift) if g is None else g
    rng = np.random.default_rng(seed + 9)
    keep = (rng.random((n, k)) < 0.4).astype(np.uint8) * rng.integers(1, 256, (n, k)).astype(np.uint8) if mask else None
    d_keep = None
    if mask:
        d_keep = torch.from_numpy(np.pad(keep, ((0, 0), (0, gap)), constant_values=1)).to(DEV)[:, :k]
    old = torch.randn((n, k + gap), device=DEV)
    out = old.clone()
    ops.weight_grad(g, x, mask=d_keep, out=out[:, :k], accumulate=accumulate)
    want, bound = Q.weight_grad(g, q, s, keep)
    if accumulate:
        want = want + Q.f64(old[:, :k])
        bound = bound + Q.U32 * np.abs(want)
        if mask:
            assert torch.equal(out[:, :k][torch.from_numpy(keep == 0).to(DEV)], old[:, :k][torch.from_numpy(keep == 0).to(DEV)])
    assert (np.abs(Q.f64(out[:, :k]) - want) <= 1.001 * bound).all()
    assert torch.equal(out[:, k:], old[:, k:])


@pytest.mark.parametrize("m", [1, 2, 31, 64, 127, 128, 129, 255, 257, 600, 2049, 8193, 20000])
def test_gradient_rows(ops, m):
    check_gradient(ops, m, 40, 70, "fp32", seed=m)
    check_gradient(ops, m, 65, 33, "bf16", seed=m, mask=True, gap=1, shift=1)


@pytest.mark.parametrize("n", EDGES)
def test_gradient_columns(ops, n):
    check_gradient(ops, 150, n, 66, "fp16", seed=n, accumulate=True)
    check_gradient(ops, 90, 37, n, "bf16", seed=n, mask=True, accumulate=True, gap=5)


@pytest.mark.parametrize("m,n,k", [(64, 512, 512), (1000, 700, 900), (300, 1500, 100), (40, 100, 3000), (4100, 260, 520),
                                   (128, 2500, 2600), (700, 20, 5000), (100, 2400, 2410), (30, 4300, 4301),
                                   (256, 1500, 1401), (256, 1400, 1300)])
def test_gradient_sizes(ops, m, n, k):
    for dtype in Q.DTYPES:
        check_gradient(ops, m, n, k, dtype, seed=m, mask=dtype != "fp32")


def test_gradient_longest_sums(ops):
    m = S.SHIFTER_Q8_MAX_SUM
    check_gradient(ops, m, 3, 5, "fp32", g=torch.ones((m, 3), device=DEV), ends=True)
    g = torch.full((m, 2), -1.0, device=DEV)
    x = Q8Matrix(torch.full((m, 16), -128, dtype=torch.int8, device=DEV), torch.ones(m, device=DEV), 3)
    d = ops.weight_grad(g, x)
    assert (torch.abs(d - 128.0 * m) <= 128.0 * m * 2.0 ** -21).all()
    for call in (lambda: S.shifter_weight_grad_q8_layout(m + 1, 2, 3),
                 lambda: S.shifter_weight_grad_q8(ops.ctx, g, 0, 2, x.q, 16, x.scale, m + 1, 2, 3, None, 0, 0, d, 3, ops.work, 1 << 40)):
        with pytest.raises(S.ShifterError) as e:
            call()
        assert e.value.code == S.SHIFTER_ERR_CAPACITY


def test_gradient_magnitudes(ops):
    """Columns from the smallest numbers to the largest side by side, columns of zeros, one row far above
    the others, rows whose scale is zero."""
    m, n, k = 300, 70, 45
    e = torch.linspace(-120, 100, n, dtype=torch.float64)
    g = (torch.randn(m, n, dtype=torch.float64, generator=torch.Generator().manual_seed(1)) * 2.0 ** e).float()
    g[:, 5] = 0
    g[17] *= 2.0 ** 14
    g = g.to(DEV)
    x, q, s = matrix(m, k, 7)
    x.scale[3:40] = 0
    s[3:40] = 0
    got = ops.weight_grad(g, x)
    want, bound = Q.weight_grad(g, q, s)
    # p below the normal numbers is held in steps of 2^-149: its own rounding
    bound = bound + (2.0 ** -149 * np.abs(q.astype(np.float64)).sum(0))[None, :]
    assert (np.abs(Q.f64(got) - want) <= 1.001 * bound).all()
    assert (got[5] == 0).all()


def test_gradient_not_finite(ops):
    for value in (float("nan"), float("inf"), -float("inf")):
        x, q, s = matrix(200, 40, 3)
        g = grads(200, 70, "bf16", 4)
        clean = ops.weight_grad(g, x)
        g[150, 66] = value
        mask = torch.ones((70, 40), dtype=torch.uint8, device=DEV)
        mask[66, 5] = 0
        d = ops.weight_grad(g, x, mask=mask)
        assert torch.isnan(d[66][mask[66] != 0]).all() and d[66, 5] == 0
        assert torch.equal(torch.cat([d[:66], d[67:]]), torch.cat([clean[:66], clean[67:]]))
    x.scale[9] = float("nan")               # a token that could not be coded: every column has it
    assert torch.isnan(ops.weight_grad(g, x)).all()


def test_gradient_no_rows(ops):
    x = Q8Matrix(torch.zeros((0, 16), dtype=torch.int8, device=DEV), torch.zeros(0, device=DEV), 9)
    g = torch.zeros((0, 11), device=DEV)
    assert (ops.weight_grad(g, x) == 0).all()
    out = torch.randn((11, 9), device=DEV)
    old = out.clone()
    assert torch.equal(ops.weight_grad(g, x, out=out, accumulate=True), old)
    assert ops.weight_grad(torch.zeros((5, 0), device=DEV), matrix(5, 9, 1)[0]).shape == (0, 9)


def test_refusals(ops):
    a, _, _ = matrix(4, 40, 1)
    b, _, _ = matrix(6, 40, 2)
    with pytest.raises(ValueError):
        ops.matmul(a, matrix(6, 41, 2)[0])
    for kw in (dict(bias=torch.zeros(5, device=DEV)), dict(bias=torch.zeros(6)), dict(dtype=torch.float64),
               dict(out=torch.zeros((4, 7), device=DEV)), dict(out=torch.zeros((6, 4), device=DEV).t())):
        with pytest.raises(ValueError):
            ops.matmul(a, b, **kw)
    tall, _, _ = matrix(2300, 40, 3)
    g = torch.zeros((4, 6), device=DEV)
    for kw in (dict(mask=torch.zeros((6, 39), dtype=torch.uint8, device=DEV)), dict(mask=torch.zeros((6, 40), device=DEV)),
               dict(mask=torch.zeros((6, 40), dtype=torch.uint8)), dict(accumulate=True),
               dict(out=torch.zeros((6, 40), device=DEV, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            ops.weight_grad(g, a, **kw)
    with pytest.raises(ValueError):
        ops.weight_grad(torch.zeros((5, 6), device=DEV), a)
    c = torch.zeros((4, 6), device=DEV)
    call = lambda **kw: S.shifter_matmul_q8(ops.ctx, *{**dict(qa=a.q, la=48, sa=a.scale, qb=b.q, lb=48, sb=b.scale, m=4, n=6, k=40,
                                                              bias=None, flags=0, c=c, t=0, lc=6), **kw}.values())
    for kw, what in ((dict(qa=None), "NULL"), (dict(sb=None), "NULL"), (dict(c=None), "NULL"), (dict(la=40), "16 bytes"),
                     (dict(la=32), "rounded up"), (dict(lc=5), "stride"), (dict(t=7), "element type"), (dict(flags=2), "flag"),
                     (dict(m=1 << 31), "2^31"), (dict(lb=(1 << 22) + 16), "2^22")):
        with pytest.raises(S.ShifterError) as e:
            call(**kw)
        assert e.value.code == S.SHIFTER_ERR_INVALID_ARG and what in str(e.value), kw
    work = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    d = torch.zeros((6, 40), device=DEV)
    for w, n, what in ((work, 100, "too small"), (None, 1 << 20, "256"), (work[1:], 1 << 19, "256")):
        with pytest.raises(S.ShifterError) as e:
            S.shifter_weight_grad_q8(ops.ctx, torch.zeros((2300, 6), device=DEV), 0, 6, tall.q, 48, tall.scale, 2300, 6, 40,
                                     None, 0, 0, d, 40, w, n)
        assert e.value.code == S.SHIFTER_ERR_INVALID_ARG and what in str(e.value)


# ---- used together ------------------------------------------------------------------------

def test_recorded_graph():
    """Norm, product, quantise, product and gradient recorded once and replayed on new inputs, with eager
    calls of the same handle and waits between the replays."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ops = Q8()
        gen = torch.Generator(device=DEV).manual_seed(1)
        rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
        w1, w2 = ops.quantize(rand(200, 130)), ops.quantize(rand(130, 200))
        x, r, g, nw = rand(90, 130).bfloat16(), rand(90, 130).bfloat16(), rand(90, 200).bfloat16(), 1 + 0.1 * rand(130)

        def step():
            m, h = ops.rms_norm(x, nw, 1e-6, residual=r)
            u = ops.matmul(m, w1, relu=True)
            y = ops.matmul(ops.quantize(u), w2, dtype=torch.float32)
            return h, u, y, ops.weight_grad(g, m), ops.dequantize(m)

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            recorded = step()
        for i in range(4):
            for t in (x, r, g):
                t.copy_(rand(*t.shape))
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(recorded, step()):
                assert torch.equal(a, b)
            big = rand(3000, 200)                          # an eager call that outgrows the workspace
            ops.weight_grad(big, ops.quantize(rand(3000, 130 + i)))
        torch.cuda.synchronize()
        ops.close()


def test_checkpointed_linear(ops):
    """Forward as torch's, x's gradient as torch's, the weights' gradient that of the 8-bit input and zero
    where the mask is."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(50, 70, generator=gen, device=DEV, requires_grad=True)
    w = torch.randn(30, 70, generator=gen, device=DEV, requires_grad=True)
    mask = (torch.rand(30, 70, generator=gen, device=DEV) < 0.5).to(torch.uint8)
    y = checkpointed_linear(x, w, ops, mask)
    assert torch.equal(y, x.detach() @ w.detach().t())
    g = torch.randn(30, 50, generator=gen, device=DEV).t()       # not the usual order
    y.backward(g)
    assert torch.equal(x.grad, g.contiguous() @ w.detach())
    q, s = Q.quantize(x)
    want, bound = Q.weight_grad(g, q, s.astype(np.float32), mask.cpu().numpy())
    assert (np.abs(Q.f64(w.grad) - want) <= 1.001 * bound).all()
    # near the gradient of the input as it was: codes are half a unit off at most
    full = Q.f64(g).T @ Q.f64(x) * (mask.cpu().numpy() != 0)
    off = np.abs(Q.f64(g)).T @ (0.5 * s[:, None] * np.ones((1, 70)))
    assert (np.abs(Q.f64(w.grad) - full) <= 1.001 * off + bound + 1e-6 * np.abs(full)).all()
    # an expanded gradient (that of a sum) and bf16
    x16, w16 = x.detach().bfloat16().requires_grad_(), w.detach().bfloat16().requires_grad_()
    checkpointed_linear(x16, w16, ops).sum().backward()
    assert w16.grad.dtype == torch.bfloat16 and torch.isfinite(w16.grad).all()
