"""The 8-bit operators' handle without a GPU: which stream and device it is tied to."""
import ctypes
import types

import pytest
import torch

from paper_2309_06973_amd import q8, shifter as S


@pytest.fixture
def device(monkeypatch):
    """A device that is not there, its current stream .stream."""
    now = types.SimpleNamespace(stream=7)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "set_device", lambda d: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: types.SimpleNamespace(cuda_stream=now.stream))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(q8, "_raw_stream", lambda index: now.stream)
    monkeypatch.setattr(q8, "load_calls", lambda: None)
    monkeypatch.setattr(S, "load_library", lambda: types.SimpleNamespace(shifter_create=lambda *a: 0))
    return now


def context(device, stream):
    c = S.shifter_create(device, stream)
    c.handle = ctypes.c_void_p(1)
    return c


def test_a_given_context_says_the_stream(device):
    ctx = context(0, 7)
    device.stream = 9
    ops = q8.Q8(ctx=ctx)                       # made under another stream than the context's
    with pytest.raises(RuntimeError, match="stream"):
        ops._enter()
    device.stream = 7
    assert ops._enter() == (1, 0)
    assert context(0, None).stream == 0        # the default stream


def test_a_given_context_says_the_device(device):
    with pytest.raises(ValueError, match="device"):
        q8.Q8(device=1, ctx=context(0, 7))
    assert q8.Q8(device=1, ctx=context(1, 7))._enter() == (1, 1)


@pytest.mark.gpu
def test_a_pipelines_context():
    """The handle of a context runs on the context's stream, whatever stream it is made under."""
    stream = torch.cuda.Stream()
    ctx = S.shifter_create(0, stream.cuda_stream)
    ops = q8.Q8(ctx=ctx)
    x = torch.randn(40, 70, device="cuda")
    with pytest.raises(RuntimeError, match="stream"):
        ops.quantize(x)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        m = ops.quantize(x)
    torch.cuda.synchronize()
    there = q8.Q8()
    assert torch.equal(m.q, there.quantize(x).q)
    torch.cuda.synchronize()
    there.close()
    ops.close()                                # leaves the context
    S.shifter_destroy(ctx)


@pytest.mark.parametrize("recording", [False, True])
def test_a_workspace_is_as_large_as_asked_for(device, monkeypatch, recording):
    """Another host thread that puts a smaller one in the place of a call's workspace, right behind its allocation, does not
    leave the call with less than it asked for."""
    made = lambda n, **kw: types.SimpleNamespace(numel=lambda: n)

    class Interrupted(q8.Q8):
        @property
        def work(self):
            return self.held

        @work.setter
        def work(self, w):
            self.held = w and made(10)

    class Recorded(list):
        def append(self, w):
            super().append(w)
            super().append(made(10))

    ops = Interrupted(ctx=context(0, 7))
    ops.recorded = Recorded()
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: recording)
    monkeypatch.setattr(torch, "empty", made)
    assert ops._room(100).numel() == 100


@pytest.mark.gpu
def test_two_threads():
    """Gradients of two host threads on one handle: a call's launches follow one another."""
    import threading
    ops = q8.Q8()
    g = torch.Generator(device="cuda").manual_seed(1)
    pairs = [(torch.randn(m, n, generator=g, device="cuda"), ops.quantize(torch.randn(m, k, generator=g, device="cuda")))
             for m, n, k in ((2500, 300, 200), (2700, 290, 310))]
    want = [ops.weight_grad(a, b) for a, b in pairs]
    got, failed = [[], []], []

    def work(i):
        try:
            for _ in range(100):
                got[i].append(ops.weight_grad(*pairs[i]))
        except Exception as e:                 # pragma: no cover
            failed.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    assert all(torch.equal(d, want[i]) for i in range(2) for d in got[i])
    ops.close()
