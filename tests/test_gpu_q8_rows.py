"""Rows to 8 bits and back, and the RMS norm with an 8-bit output, against their definition in
64 bits.

Codes and the residual stream are whole decisions and compared exactly.  Scales: a / 127 is one
correctly rounded division, half a step (2^-24) of fp32; the norm's is worked out in 64 bits and
rounded once, and the sum in 64 bits is off by less than 2^-40 of it: both are allowed 1.5 half
steps plus half the smallest number.  Values read back: code * scale is one fp32 rounding, then
half a step of the element type."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as Q
from paper_2309_06973_amd import shifter as S
from paper_2309_06973_amd.q8 import Q8, Q8Matrix

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ops():
    o = Q8()
    yield o
    torch.cuda.synchronize()
    o.close()


def make(rows, cols, dtype, seed, gap=0, shift=0):
    """A view of a larger buffer: `gap` elements between rows, the first `shift` elements in."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows * (cols + gap) + shift, generator=g)
    x *= torch.exp(torch.randn(x.shape, generator=g))
    x = x.to(Q.DTYPES[dtype]).to(DEV)
    return x[shift:].view(rows, cols + gap)[:, :cols]


def check_scales(got, want, where=""):
    got, want = got.cpu().numpy().astype(np.float64), np.asarray(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), where
    ok = ~np.isnan(want)
    assert (np.abs(got[ok] - want[ok]) <= 1.5 * Q.U32 * want[ok] + Q.TINY32 / 2).all(), where


def check_codes(m, want):
    q = m.q.cpu().numpy()
    assert np.array_equal(q[:, :m.cols], want)
    pad = -(-m.cols // 16) * 16
    assert (q[:, m.cols:pad] == 0).all()


def check_values(ops, m, dtype):
    got = Q.f64(ops.dequantize(m, Q.DTYPES[dtype]))
    s = m.scale.cpu().numpy().astype(np.float64)
    want = m.q[:, :m.cols].cpu().numpy().astype(np.float64) * s[:, None]
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert (np.abs(got[ok] - want[ok]) <= (Q.HALF_STEP[dtype] + 1.01 * Q.U32) * np.abs(want[ok]) + 1.01 * Q.LEAST[dtype]).all()


COLS = [1, 2, 7, 8, 9, 15, 16, 17, 100, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1024, 1025, 2047, 2048, 2049, 4096, 4097, 8192, 8193,
        16384, 16385, 32768, 32769, 50001]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("cols", COLS)
def test_quantize(ops, cols, dtype):
    for rows, gap, shift, relu in ((1, 0, 0, False), (5, 0, 1, True), (6, 3, 0, False)):
        print(f"quantize rows={rows} cols={cols} gap={gap} shift={shift} relu={relu} {dtype}", flush=True)
        x = make(rows, cols, dtype, cols + rows, gap, shift)
        m = ops.quantize(x, relu=relu)
        q, s = Q.quantize(x, relu)
        check_codes(m, q)
        check_scales(m.scale, s)
        check_values(ops, m, dtype)


@pytest.mark.parametrize("rows,cols", [(0, 7), (3, 0), (0, 0), (1000, 40), (777, 130),
                                       (9000, 700), (9001, 1100), (2500, 4000), (300, 3001), (300, 8000), (600, 9000), (9, 2000),
                                       (70001, 3), (66000, 200), (17000, 300)])
def test_quantize_shapes(ops, rows, cols):
    x = make(rows, cols, "bf16", 3)
    m = ops.quantize(x)
    q, s = Q.quantize(x)
    check_codes(m, q)
    check_scales(m.scale, s)
    assert ops.dequantize(m).shape == (rows, cols)


def test_ties_and_ends(ops):
    """Quotients exactly between two codes, for many largest values; in every type."""
    top = torch.tensor([2.0, 254.0, 127.0, 0.5, 1.0, 3.0, 2.0 ** -14, 96.0])
    half = torch.arange(-127, 128).float()
    x = torch.cat([half[None, :] * (top[:, None] / 254.0), top[:, None], -top[:, None] / 2], 1)
    for dtype in Q.DTYPES:
        y = x.to(Q.DTYPES[dtype]).to(DEV)
        m = ops.quantize(y)
        check_codes(m, Q.quantize(y)[0])
    # the values around every tie, one step of fp32 either way
    a = torch.tensor([1.0, 1.7, 3.1e-5, 7.7e20])
    t = (torch.arange(-127, 127).float() + 0.5)
    for nudge in (-1, 0, 1):
        x = (t[None, :].double() * a[:, None].double() / 127.0).float()
        x = torch.cat([(x.view(torch.int32) + nudge).view(torch.float32), a[:, None]], 1).to(DEV)
        check_codes(ops.quantize(x), Q.quantize(x)[0])


def test_far_magnitudes(ops):
    """Largest values from the smallest number there is to the largest; zero rows; signs of zero."""
    rows = []
    g = torch.Generator().manual_seed(5)
    for e in (-149, -148, -140, -127, -126, -125, -110, -101, -100, -99, -60, 0, 60, 120, 127):
        r = torch.randn(64, generator=g, dtype=torch.float64)
        r = r / r.abs().max() * 2.0 ** e
        rows.append(r.float())
    rows += [torch.zeros(64), -torch.zeros(64), torch.full((64,), torch.finfo(torch.float32).max)]
    x = torch.stack(rows).to(DEV)
    m = ops.quantize(x)
    q, s = Q.quantize(x)
    check_codes(m, q)
    check_scales(m.scale, s)
    assert (m.scale[-3:-1] == 0).all()


def test_rows_that_are_not_finite(ops):
    inf, nan = float("inf"), float("nan")
    for dtype in Q.DTYPES:
        for cols in (33, 700, 5000, 40000):
            x = make(6, cols, dtype, 8)
            x[0, cols // 2] = nan
            x[1, cols - 1] = inf
            x[2, 0] = -inf
            x[4] = 0
            for relu in (False, True):
                m = ops.quantize(x, relu=relu)
                q, s = Q.quantize(x, relu)
                check_codes(m, q)
                check_scales(m.scale, s)
                bad = torch.isnan(ops.dequantize(m)).all(1).cpu().tolist()
                assert bad == [True, True, not relu, False, False, False]


def test_what_lies_behind_the_rows_is_left(ops):
    for cols in (5, 16, 30):
        pad = -(-cols // 16) * 16
        buf = torch.full((4, pad + 32), 77, dtype=torch.int8, device=DEV)
        m = Q8Matrix(buf, torch.zeros(4, device=DEV), cols)
        ops.quantize(make(4, cols, "fp32", 2), out=m)
        assert (buf[:, pad:] == 77).all() and (buf[:, cols:pad] == 0).all()
        out = torch.full((4, cols + 3), 9.0, device=DEV)
        ops.dequantize(m, out=out[:, :cols])
        assert (out[:, cols:] == 9.0).all()


def test_many_rows(ops):
    """More rows than one round of blocks."""
    rows = (1 << 23) + 9
    x = torch.randn(rows, 1, device=DEV, dtype=torch.bfloat16)
    m = ops.quantize(x)
    assert torch.equal(m.q[:, 0].float(), 127 * torch.sign(x[:, 0].float()))
    assert torch.equal(m.scale, (x[:, 0].double().abs() / 127).float())     # in 64 bits: torch's 32-bit one multiplies
    y = ops.dequantize(m, torch.bfloat16)
    assert torch.equal(y[-9:], (m.q[-9:, :1].float() * m.scale[-9:, None]).bfloat16())


def test_far_offsets(ops):
    """Elements, codes and values more than 2^32 bytes (and elements) from the first."""
    rows, ld = 1040, 1 << 22
    buf = torch.empty(rows * ld, dtype=torch.float16, device=DEV)
    x = buf.view(rows, ld)[:, :333]
    x.copy_(make(rows, 333, "fp16", 4))
    q = torch.empty((rows, ld), dtype=torch.int8, device=DEV)
    m = Q8Matrix(q, torch.empty(rows, device=DEV), 333)
    ops.quantize(x, out=m)
    want, s = Q.quantize(x)
    assert np.array_equal(q[:, :333].cpu().numpy(), want)
    check_scales(m.scale, s)
    h = buf.view(rows, ld)[:, 1000:1333]
    ops.dequantize(m, out=h)
    assert torch.equal(h, ops.dequantize(m, torch.float16))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("cols", COLS)
def test_rms_norm(ops, cols, dtype):
    w = (1.0 + 0.3 * torch.randn(cols + 1, generator=torch.Generator().manual_seed(cols))).to(DEV)[1:]
    for rows, gap, shift, res in ((1, 0, 0, True), (5, 0, 1, False), (6, 5, 0, True)):
        print(f"rms_norm rows={rows} cols={cols} gap={gap} shift={shift} residual={res} {dtype}", flush=True)
        x = make(rows, cols, dtype, cols + rows, gap, shift)
        r = make(rows, cols, dtype, cols + rows + 1, 2 * gap, 0) if res else None
        m, h = ops.rms_norm(x, w, 1e-5, residual=r)
        q, s, want_h = Q.rms_norm(x, w, float(np.float32(1e-5)), r)
        assert torch.equal(h.cpu(), want_h)
        check_codes(m, q)
        check_scales(m.scale, s)
        # in place, in both operands
        if res:
            for at in (0, 1):
                a, b = x.clone(), r.clone()
                m2, h2 = ops.rms_norm(a, w, 1e-5, residual=b, h=(a, b)[at])
                assert h2 is (a, b)[at] and torch.equal(h2.cpu(), want_h)
                assert torch.equal(m2.q, m.q) and torch.equal(m2.scale, m.scale)


@pytest.mark.parametrize("rows,cols", [(70001, 3), (66000, 150), (17000, 300), (9000, 700), (9001, 1100), (2500, 4000), (300, 3001), (300, 8000), (600, 9000),
                                       (9, 2000), (530, 20000)])
def test_rms_norm_many_rows(ops, rows, cols):
    """More rows than a launch's blocks hold at once, and both sides of the rules on rows."""
    for dtype in Q.DTYPES:
        x, r = make(rows, cols, dtype, 1), make(rows, cols, dtype, 2, gap=3)
        w = (1.0 + 0.3 * torch.randn(cols, generator=torch.Generator().manual_seed(3))).to(DEV)
        q, s, want_h = Q.rms_norm(x, w, float(np.float32(1e-6)), r)
        m, h = ops.rms_norm(x, w, 1e-6, residual=r, h=x)          # in place
        assert h is x and torch.equal(h.cpu(), want_h)
        check_codes(m, q)
        check_scales(m.scale, s)


def test_rms_norm_ends(ops):
    """Zero rows (with and without eps), weights that are zero, values whose squares leave 32 bits,
    rows that are not finite, sums that overflow the element type, no columns."""
    inf, nan = float("inf"), float("nan")
    for dtype in Q.DTYPES:
        for cols in (24, 3000, 40000):
            x = make(8, cols, dtype, 6)
            w = torch.ones(cols, device=DEV)
            w[::3] = 0.0
            x[0] = 0
            x[1, 3] = nan
            x[2, cols - 1] = inf
            x[3, 0] = inf                     # under a weight of zero: no number either
            if dtype == "fp32":
                x[4] *= 1e19
                x[5] *= 1e-25
            r = torch.zeros_like(x)
            big = float(torch.finfo(x.dtype).max)
            x[6, 1], r[6, 1] = big, big       # the stream overflows
            for eps in (0.0, 1e-6):
                m, h = ops.rms_norm(x, w, eps, residual=r)
                with np.errstate(all="ignore"):
                    q, s, want_h = Q.rms_norm(x, w, float(np.float32(eps)), r)
                assert torch.equal(torch.nan_to_num(h.cpu(), 1, 2, 3), torch.nan_to_num(want_h, 1, 2, 3))
                check_codes(m, q)
                check_scales(m.scale, s, (dtype, cols, eps))
                assert m.scale[0] == 0
    m, h = ops.rms_norm(make(3, 0, "bf16", 1), torch.empty(0, device=DEV), 1e-6)
    assert (m.scale == 0).all()
    m, h = ops.rms_norm(make(0, 50, "bf16", 1), torch.ones(50, device=DEV), 1e-6, residual=make(0, 50, "bf16", 1))
    assert h.shape == (0, 50)


def test_refusals(ops):
    x = make(4, 32, "bf16", 1)
    w = torch.ones(32, device=DEV)
    for bad in (x.double(), x.cpu(), x.t(), x[0], x[:, ::2]):
        with pytest.raises(ValueError):
            ops.quantize(bad)
    with pytest.raises(ValueError):
        ops.quantize(x, out=ops.quantize(make(4, 31, "bf16", 1)))
    for kw in (dict(residual=x.float()), dict(residual=x[:3]), dict(h=x), dict(residual=x, h=x.float())):
        with pytest.raises(ValueError):
            ops.rms_norm(x, w, 1e-6, **kw)
    for bad in (w[:31], w.double(), w.cpu()):
        with pytest.raises(ValueError):
            ops.rms_norm(x, bad, 1e-6)
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(S.ShifterError) as e:
            ops.rms_norm(x, w, eps)
        assert e.value.code == S.SHIFTER_ERR_INVALID_ARG and "eps" in str(e.value)
    q, s = torch.empty((4, 32), dtype=torch.int8, device=DEV), torch.empty(4, device=DEV)
    call = lambda *a: S.shifter_quantize_q8(ops.ctx, *a)
    for args, what in (((x, 3, 32, 4, 32, 0, q, 32, s), "element type"), ((x, 1, 32, 4, 32, 2, q, 32, s), "flag"),
                       ((x, 1, 31, 4, 32, 0, q, 32, s), "stride"), ((None, 1, 32, 4, 32, 0, q, 32, s), "NULL"),
                       ((x, 1, 32, 4, 32, 0, q, 24, s), "16 bytes"), ((x, 1, 32, 4, 32, 0, q, 16, s), "rounded up"),
                       ((x, 1, 32, 4, 32, 0, None, 32, s), "NULL"), ((x, 1, 32, 4, 32, 0, q, 32, None), "NULL"),
                       ((x, 1, 32, 1 << 31, 32, 0, q, 32, s), "2^31")):
        with pytest.raises(S.ShifterError) as e:
            call(*args)
        assert e.value.code == S.SHIFTER_ERR_INVALID_ARG and what in str(e.value), args
    with torch.cuda.stream(torch.cuda.Stream()):
        with pytest.raises(RuntimeError, match="stream"):
            ops.quantize(x)
