"""Log probabilities, entropies, alternatives and their gradient against their definition in 64 bits.  Columns of
alternatives are whole decisions and compared exactly; how far numbers may be off is derived in oracle.learn_oracle."""
import numpy as np
import pytest
import torch

from oracle import learn_oracle as L
from paper_2309_06973_amd import shifter as S
from paper_2309_06973_amd.q8 import Q8, target_log_probs

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


def make(rows, cols, dtype, seed, gap=0, shift=0, size=3.0):
    """A view of a larger buffer: `gap` elements between rows, the first `shift` elements in."""
    g = torch.Generator().manual_seed(seed)
    x = (size * torch.randn(rows * (cols + gap) + shift, generator=g)).to(dtype).to(DEV)
    return x[shift:].view(rows, cols + gap)[:, :cols]


def targets(rows, cols, seed):
    return torch.randint(0, max(1, cols), (rows,), generator=torch.Generator().manual_seed(seed)).to(DEV)


def near(got, want, off, what):
    got = got.detach().cpu().double().numpy()
    want, off = np.asarray(want), np.asarray(off)
    assert got.shape == want.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    same = np.isinf(want)
    assert np.array_equal(got[same], want[same]), what
    ok = np.isfinite(want)
    bad = np.abs(got[ok] - want[ok]) > np.broadcast_to(off, want.shape)[ok]
    assert not bad.any(), (what, got[ok][bad][:3], want[ok][bad][:3], np.broadcast_to(off, want.shape)[ok][bad][:3])


def check(r, x, target, top, scale=1.0):
    ref = L.Logs(x, scale)
    near(r.lse, ref.lse, ref.rel + L.U * np.abs(ref.lse), "lse")
    if target is not None:
        want = ref.logp(target)
        near(r.logp, want, ref.rel + L.U * np.abs(want), "logp")
    if r.entropy is not None:
        near(r.entropy, ref.entropy, ref.off_h + L.U * np.abs(ref.entropy), "entropy")
    if top:
        index = ref.top(top)
        assert np.array_equal(r.index.cpu().numpy(), index)
        want = np.take_along_axis(ref.log_p, index, 1)
        near(r.top, want, ref.rel[:, None] + L.U * np.abs(want), "top")
    return ref


COLS = [1, 2, 7, 8, 9, 16, 17, 63, 64, 127, 128, 129, 200, 255, 256, 257, 511, 512, 513, 1000, 1024, 1025, 2047, 2048, 2049, 4097, 8192, 8193,
        16391, 50001, 131072]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", COLS)
def test_log_probs(ops, cols, dtype):
    for rows, gap, shift, top, entropy, scale in ((1, 0, 0, 5, True, 1.0), (5, 0, 1, 0, True, 0.7), (6, 3, 0, 20, False, 1.25), (37, 1, 3, 32, True, 1.0),
                                                  (3, 0, 0, 1, False, 1.0), (2, 8, 5, 0, False, 2.5)):
        top = min(top, cols)
        print(f"log_probs rows={rows} cols={cols} gap={gap} shift={shift} top={top} entropy={entropy} scale={scale} {dtype}", flush=True)
        x, t = make(rows, cols, dtype, cols + rows, gap, shift), targets(rows, cols, rows)
        r = ops.log_probs(x, t, scale=scale, entropy=entropy, top=top)
        assert (r.entropy is None) == (not entropy) and (r.top is None) == (not top)
        check(r, x, t, top, scale)


@pytest.mark.parametrize("rows, cols, top", [(0, 7, 2), (700, 40, 8), (700, 40, 9), (3000, 130, 3), (777, 3000, 4), (513, 9000, 20), (511, 9000, 20),
                                             (100, 20000, 32), (9, 262147, 32), (1, 1000003, 32), (70001, 3, 3)])
def test_shapes(ops, rows, cols, top):
    x, t = make(rows, cols, torch.bfloat16, 3), targets(rows, cols, 5)
    check(ops.log_probs(x, t, entropy=True, top=top), x, t, top)


def test_no_columns_and_no_targets(ops):
    r = ops.log_probs(torch.zeros(3, 0, device=DEV), torch.tensor([-1, 0, 5], device=DEV), entropy=True)
    assert r.lse.tolist() == [-INF] * 3 and torch.isnan(r.entropy).all()
    assert r.logp[0] == 0 and torch.isnan(r.logp[1:]).all()
    x = make(5, 300, torch.float16, 4)
    r = ops.log_probs(x)
    assert r.logp is None and r.entropy is None and r.top is None and r.index is None
    check(r, x, None, 0)


@pytest.mark.parametrize("cols", [5, 100, 900, 3000, 20000])
def test_targets_that_are_left_out_or_outside(ops, cols):
    x = make(6, cols, torch.float32, 1)
    t = torch.tensor([-1, -100, cols, 1 << 40, -(1 << 60), cols - 1], device=DEV)
    r = ops.log_probs(x, t)
    check(r, x, t, 0)
    assert r.logp[:2].tolist() == [0, 0] and torch.isnan(r.logp[2:4]).all() and r.logp[4] == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [33, 200, 700, 5000, 20000, 70000])
def test_places_that_are_masked(ops, cols, dtype):
    """Minus infinity, the type's lowest value, rows with hardly anything or nothing left, infinity and NaN."""
    lowest = torch.finfo(dtype).min
    x = make(9, cols, dtype, 7)
    x[0, ::2] = -INF
    x[1, 1:] = -INF                             # one left
    x[2] = -INF                                 # nothing left
    x[2, cols - 1] = -INF
    x[3] = lowest                               # all alike
    x[4, : cols // 2] = lowest
    x[5, cols // 3] = NAN
    x[6, cols - 1] = INF
    x[7] = -INF
    x[7, cols // 2] = lowest
    x[8] = 1.5                                  # ties
    t = torch.tensor([1, 0, 0, 3, cols - 1, 0, 0, cols // 2, 5], device=DEV)
    top = min(20, cols)
    r = ops.log_probs(x, t, entropy=True, top=top)
    check(r, x, t, top)
    assert r.logp[1] == 0 and r.entropy[1] == 0 and r.lse[2] == -INF
    assert r.index[2].tolist() == list(range(top)) and r.index[3].tolist() == list(range(top))
    assert torch.isnan(r.lse[5:7]).all() and torch.isnan(r.logp[5:7]).all()


@pytest.mark.parametrize("cols", [200, 1000, 8000, 50000, 300000])
def test_alternatives_in_every_order(ops, cols):
    """Rising and falling rows, rows of few values, and signs of zero: where many places reach any bound."""
    i = torch.arange(cols, device=DEV)
    rows = [i, -i, i % 7, -(i % 1001), (i * 7919) % cols, (i // 8) % 64, (i // 512) * 1.0, -((i // 8) % 2048) * 1.0]
    zeros = torch.zeros(cols, device=DEV)
    zeros[1::2] = -0.0
    rows += [zeros, torch.where(i < cols // 2, -1.0, 0.0), torch.where(i % 3 == 0, -INF, -5.0)]
    x = torch.stack([r.float() for r in rows]) * 0.01
    for top in (1, 8, 9, 32):
        for dtype in (torch.float32, torch.bfloat16):
            y = x.to(dtype)
            r = ops.log_probs(y, None, top=top)
            assert np.array_equal(r.index.cpu().numpy(), L.Logs(y).top(top)), (top, dtype)


def test_far_values(ops):
    """Logits at the ends of fp32, and scales that take them out of it."""
    x = torch.tensor([[3e38, -3e38, 1.0, 3e38], [1e-40, -1e-40, 0.0, 0.0], [80.0, -80.0, 0.0, 100.0], [1e30, 1e30, 0.0, -1e30]], device=DEV)
    t = torch.tensor([1, 0, 1, 0], device=DEV)
    for scale in (1.0, 2.0 ** -20):
        r = ops.log_probs(x, t, scale=scale, entropy=True, top=4)
        ref = L.Logs(x, scale)
        with np.errstate(over="ignore"):
            near(r.lse, ref.lse, ref.rel + L.U * np.abs(ref.lse), "lse")
        near(r.entropy, ref.entropy, ref.off_h + L.U, "entropy")
        assert np.array_equal(r.index.cpu().numpy(), ref.top(4))


def test_the_same_every_time(ops):
    x, t = make(3, 100001, torch.float16, 9), targets(3, 100001, 9)
    a = ops.log_probs(x, t, entropy=True, top=20)
    for _ in range(20):
        b = ops.log_probs(x, t, entropy=True, top=20)
        ops.log_probs(x[:1, :30000], t[:1], top=7)                 # other sizes in the same workspace
        assert all(torch.equal(p, q) for p, q in zip(a, b))


# ---- the gradient
def check_grad(got, ref, dtype, target, **g):
    want, off = ref.grad(target, **g)
    near(got, want, off + L.HALF_STEP[dtype] * (np.abs(want) + off) + L.LEAST[dtype], "grad")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", COLS)
def test_gradient(ops, cols, dtype):
    for rows, gap, shift, which, scale in ((1, 0, 0, "p", 1.0), (5, 0, 1, "pe", 0.7), (6, 3, 0, "pel", 1.25), (7, 1, 3, "l", 1.0), (3, 0, 0, "e", 1.0)):
        print(f"log_probs_grad rows={rows} cols={cols} gap={gap} shift={shift} {which} scale={scale} {dtype}", flush=True)
        x, t = make(rows, cols, dtype, cols + rows, gap, shift), targets(rows, cols, rows)
        t[0] = -1 if rows > 1 else t[0]
        ref = L.Logs(x, scale)
        g = torch.randn(3, rows, generator=torch.Generator().manual_seed(rows)).to(DEV) * 100.0
        some = dict(g_logp=g[0] if "p" in which else None, g_entropy=g[1] if "e" in which else None, g_lse=g[2] if "l" in which else None)
        norm, h = (torch.from_numpy(v).float().to(DEV) for v in (ref.norm, ref.entropy))
        wide = torch.full((rows, cols + 5), 7.0, dtype=dtype, device=DEV)
        got = ops.log_probs_grad(x, t, norm, entropy=h, scale=scale, out=wide[:, 2:cols + 2], **some)
        check_grad(got, ref, dtype, t, **some)
        assert (wide[:, :2] == 7).all() and (wide[:, cols + 2:] == 7).all()
        y = x.clone()
        assert torch.equal(ops.log_probs_grad(y, t, norm, entropy=h, scale=scale, out=y, **some), got)      # in place


def test_gradient_of_masked_rows(ops):
    for cols in (100, 900, 3000, 20000):
        x = make(6, cols, torch.float32, 2)
        x[0, ::3] = -INF
        x[1] = NAN                                  # a padded position: it is left out
        x[2] = -INF
        x[3, 5] = NAN
        x[4, 1:] = -INF
        t = torch.tensor([1, -1, -1, 0, 0, cols], device=DEV)
        r = ops.log_probs(x, t, entropy=True)
        one = torch.full((6,), -0.5, device=DEV)
        got = ops.log_probs_grad(x, t, r.norm, g_logp=one)
        assert (got[1:3] == 0).all() and torch.isnan(got[3]).all() and torch.isnan(got[5]).all()
        assert (got[4] == 0).all() and (got[0, ::3] == 0).all() and torch.isfinite(got[0]).all()
        low = torch.full((2, cols), torch.finfo(torch.float32).min, device=DEV)      # nothing left but the type's lowest value
        low_r = ops.log_probs(low, t[:2].clamp(min=0))
        d = ops.log_probs_grad(low, t[:2], low_r.norm, g_logp=one[:2] * 0, g_lse=torch.ones(2, device=DEV))
        assert ((d - 1 / cols).abs() <= 16 * np.log(cols) * L.U / cols).all()
        h = torch.ones(6, device=DEV)
        got = ops.log_probs_grad(x, t, r.norm, g_logp=one, entropy=r.entropy, g_entropy=h)
        assert torch.isfinite(got[0]).all() and (got[4].abs() <= L.U).all() and torch.isnan(got[1]).all()


@pytest.mark.parametrize("low", [-INF, torch.finfo(torch.float32).min, -1e30])
def test_large_entropy_gradient_of_masked_places(ops, low):
    """What has no probability gives 0, however large the entropy's gradient."""
    for cols in (100, 900, 3000):
        x, t = make(5, cols, torch.float32, 3), torch.tensor([1, -1, 2, 3, 6], device=DEV)
        x[:, 1::3] = low
        ref = L.Logs(x)
        norm, h = (torch.from_numpy(v).float().to(DEV) for v in (ref.norm, ref.entropy))
        some = dict(g_logp=torch.full((5,), -3.0, device=DEV), g_entropy=torch.tensor([1.5, -2.0, 100.0, 1e4, -1e20], device=DEV))
        got = ops.log_probs_grad(x, t, norm, entropy=h, **some)
        check_grad(got, ref, torch.float32, t, **some)
        assert (got[1:, 1::3] == 0).all() and got[0, 1] == -3 and (got[0, 4::3] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_autograd(ops, dtype):
    """Through torch's graph, leading dimensions and all; against the formula's and against differences."""
    x = make(6, 333, dtype, 11).reshape(2, 3, 333).clone().requires_grad_()
    t = targets(6, 333, 2).view(2, 3)
    t[1, 2] = -1
    logp, h, lse = target_log_probs(x, t, ops, scale=0.8)
    assert logp.shape == h.shape == lse.shape == (2, 3) and logp[1, 2] == 0
    w = torch.randn(3, 2, 3, generator=torch.Generator().manual_seed(1)).to(DEV)
    (w[0] * logp + w[1] * h + w[2] * lse).sum().backward()
    ref = L.Logs(x.view(6, 333), 0.8)
    w = w.view(3, 6)
    want, off = ref.grad(t.view(-1), w[0], w[2], w[1])
    # lse and the entropy are the kernel's own here
    more = np.abs(ref.p) * 0.8 * (ref.rel * 4 + ref.off_h)[:, None] * 4 * (1 + np.abs(np.where(ref.p == 0, 0, ref.log_p)))
    near(x.grad.view(6, 333), want, off + more + L.HALF_STEP[dtype] * np.abs(want) * 1.01 + L.LEAST[dtype], "autograd")
    if dtype == torch.float32:
        step = 2.0 ** -8
        for r, c in ((0, 0), (3, 100), (4, int(t.view(-1)[4]))):
            f = []
            for s in (step, -step):
                y = x.detach().double().cpu().view(6, 333).clone()
                y[r, c] += s
                o = L.Logs(y, 0.8)
                f.append(sum(float(a) @ b if np.ndim(a) else 0 for a, b in ()) + float(w[0].cpu().double().numpy() @ o.logp(t.view(-1)))
                         + float(w[1].cpu().double().numpy() @ o.entropy) + float(w[2].cpu().double().numpy() @ o.lse))
            # the third derivative is below 8 (|w| up to 3, |log p| up to 20 with p of order 1): step^2 / 6 of it
            assert abs((f[0] - f[1]) / (2 * step) - float(x.grad.view(6, 333)[r, c])) < 60 * step * step / 6 + 1e-5


def test_second_derivative_is_an_error(ops):
    x = make(3, 50, torch.float32, 1).clone().requires_grad_()
    logp, h, _ = target_log_probs(x, targets(3, 50, 1), ops)
    (dx,) = torch.autograd.grad(logp.sum() + h.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="no derivative"):
        dx.square().sum().backward()


def test_gradients_that_would_be_lost(ops):
    x = make(3, 50, torch.float32, 1).clone().requires_grad_()
    r = ops.log_probs(x, targets(3, 50, 1), entropy=True, top=3)
    for v in (r.logp, r.lse, r.entropy, r.top, r.norm):
        with pytest.raises(RuntimeError, match="passes no gradients on"):
            v.sum().backward()
    assert not r.index.requires_grad
    g = torch.ones(3, device=DEV, requires_grad=True)
    with pytest.raises(RuntimeError, match="passes no gradients on"):
        ops.log_probs_grad(x.detach(), targets(3, 50, 1), r.norm.detach(), g_logp=g).sum().backward()
    with pytest.raises(ValueError, match="needs a gradient"):
        ops.log_probs_grad(x.detach(), targets(3, 50, 1), r.norm.detach(), g_logp=g, out=torch.empty(3, 50, device=DEV))


def test_recorded(ops):
    """Two graphs of one handle, each replayed among eager work; a backward pass through torch's graph is refused."""
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        own = Q8()
        x, t = make(3, 50001, torch.bfloat16, 4).clone(), targets(3, 50001, 4)
        one = torch.full((3,), -1 / 3, device=DEV)
        eager = own.log_probs(x, t, entropy=True, top=20)
        dx = own.log_probs_grad(x, t, eager.norm, g_logp=one)
        torch.cuda.synchronize()
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                r = own.log_probs(x, t, entropy=True, top=20)
                d = own.log_probs_grad(x, t, r.norm, g_logp=one)
            graphs.append((g, r, d))
        for i in range(4):
            graphs.reverse()                       # the one recorded last is replayed first
            y = make(3, 50001, torch.bfloat16, 20 + i)
            x.copy_(y)
            want = own.log_probs(x, t, entropy=True, top=20)
            want_d = own.log_probs_grad(x, t, want.norm, g_logp=one)
            for g, r, d in graphs:
                g.replay()
                own.log_probs(x[:, :30000], t % 30000, top=3)
                assert all(torch.equal(a, b) for a, b in zip(r, want)) and torch.equal(d, want_d)
        leaf = x.detach().requires_grad_()
        g = torch.cuda.CUDAGraph()
        with pytest.raises(RuntimeError, match="can not be recorded"):
            with torch.cuda.graph(g, stream=stream):
                target_log_probs(leaf, t, own)
        torch.cuda.synchronize()
        own.close()


def test_offsets_beyond_32_bits(ops):
    """A row that starts 2^32 elements in."""
    cols, ld = 3000, (1 << 32) - 8
    buf = torch.empty(ld + cols, dtype=torch.float16, device=DEV)
    x = torch.as_strided(buf, (2, cols), (ld, 1))
    x.copy_(make(2, cols, torch.float16, 6))
    t = targets(2, cols, 1)
    r = ops.log_probs(x, t, entropy=True, top=5)
    ref = check(r, x, t, 5)
    one = torch.ones(2, device=DEV)
    check_grad(ops.log_probs_grad(x, t, torch.from_numpy(ref.norm).float().to(DEV), g_logp=one, out=x), ref, torch.float16, t, g_logp=one)


def test_what_the_interface_refuses(ops):
    x, v, n = torch.zeros(4, 20000, device=DEV), torch.zeros(4, device=DEV), torch.zeros(4, 2, device=DEV)
    t = torch.zeros(4, dtype=torch.int64, device=DEV)
    fine = dict(d_x=x, ld_x=20000, rows=4, cols=20000, dtype=0, scale=1.0, d_norm=n, d_lse=v, d_target=t, d_logp=v)
    need = S.shifter_log_probs_layout(4, 20000, 0)
    assert need > S.SHIFTER_LEARN_ZERO
    work = torch.zeros(need, dtype=torch.uint8, device=DEV)
    for change, what in ((dict(), "workspace too small"), (dict(d_work=work, work_bytes=need - 1), "too small"),
                         (dict(d_work=work.data_ptr() + 8, work_bytes=need), "256-byte"), (dict(dtype=5), "element type"),
                         (dict(scale=0.0), "scale"), (dict(scale=NAN), "scale"), (dict(scale=-1.0), "scale"), (dict(scale=2.0 ** 65), "scale"),
                         (dict(top=33), "32 alternatives"),
                         (dict(cols=3, top=4), "more alternatives"), (dict(ld_x=100), "stride"), (dict(d_lse=None), "NULL"),
                         (dict(d_logp=None), "NULL"), (dict(d_target=None), "without d_target"), (dict(top=2), "NULL"),
                         (dict(d_lse=v.data_ptr() + 2), "aligned")):
        with pytest.raises(S.ShifterError, match=what):
            S.shifter_log_probs(ops.ctx, **{**fine, **change})
    fine = dict(d_x=x, ld_x=20000, rows=4, cols=20000, dtype=0, scale=1.0, d_norm=n, d_target=t, d_g_logp=v, d_dx=x, ld_dx=20000)
    for change, what in ((dict(ld_dx=20001), "another stride"), (dict(d_norm=None), "NULL"), (dict(d_target=None), "without d_target"),
                         (dict(d_g_entropy=v), "NULL"), (dict(scale=INF), "scale")):
        with pytest.raises(S.ShifterError, match=what):
            S.shifter_log_probs_grad(ops.ctx, **{**fine, **change})
    S.shifter_log_probs(ops.ctx, **{**fine_forward(x, v, n, t), "d_work": work, "work_bytes": need})
    torch.cuda.synchronize()


def fine_forward(x, v, n, t):
    return dict(d_x=x, ld_x=20000, rows=4, cols=20000, dtype=0, scale=1.0, d_norm=n, d_lse=v, d_target=t,
                d_logp=torch.empty_like(v))
