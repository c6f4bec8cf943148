"""8-bit matrices next to the prune-and-compact pass: a rebuilt variant's linear layers served
in 8 bits, and 8-bit activations kept for the backward pass while a masked network trains on.

Every step runs in libshifter's HIP kernels on the stream that was current when the handle (or
the context that it was given) was made; a call's checks, its new tensors and the way into the C ABI are _q8.so's (csrc/q8_bind.cpp).
Raises if no ROCm device is visible."""
from __future__ import annotations

import importlib.machinery
import importlib.util
import os
from typing import Optional

import torch

from . import shifter as S

_CALLS_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_q8.so")
_calls = None
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)        # torch.cuda.current_stream's object costs 1.9 us, this 0.1


def _pad(cols: int) -> int:
    return -(-cols // S.SHIFTER_Q8_ALIGN) * S.SHIFTER_Q8_ALIGN


class Q8Matrix:
    """rows x cols values as int8 codes and one fp32 scale a row: value = code * scale.
    q: int8 [rows, at least cols], rows 16-byte aligned; scale: float32 [rows]."""
    __slots__ = ("q", "scale", "rows", "cols", "ld")

    def __init__(self, q: torch.Tensor, scale: torch.Tensor, cols: int):
        if q.dtype != torch.int8 or q.dim() != 2 or (q.shape[1] > 1 and q.stride(1) != 1):
            raise ValueError("q must be a two-dimensional int8 tensor with its columns side by side")
        if scale.dtype != torch.float32 or scale.dim() != 1 or not scale.is_contiguous():
            raise ValueError("scale must be a contiguous float32 vector")
        if scale.shape[0] != q.shape[0] or not 0 <= cols <= q.shape[1] or q.device != scale.device:
            raise ValueError("codes, scales and cols do not belong together")
        self.q, self.scale, self.rows, self.cols = q, scale, q.shape[0], cols
        pad = _pad(cols)
        self.ld = q.stride(0) if self.rows > 1 and cols else pad
        if self.rows and cols and q.storage_offset() + (self.rows - 1) * self.ld + pad > q.untyped_storage().nbytes():
            raise ValueError("the last row's buffer ends before its columns rounded up to 16")


def load_calls():
    """Loads _q8.so; raises if it has not been built (no fallback exists)."""
    global _calls
    if _calls is None:
        S.load_library()
        if not os.path.exists(_CALLS_PATH):
            raise RuntimeError(f"{_CALLS_PATH} is missing: build it with `python -m paper_2309_06973_amd.build`")
        loader = importlib.machinery.ExtensionFileLoader(f"{__package__}._q8", _CALLS_PATH)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader(loader.name, loader))
        loader.exec_module(module)
        module.bind(Q8Matrix, S._check)
        _calls = module
    return _calls


class Q8:
    """The 8-bit operators on one device and stream: the current one, or those of a given context.
    Matrices of elements are two-dimensional fp32, bf16 or fp16 tensors whose columns lie side by
    side; their rows may have any stride.
    Results are new tensors unless ``out`` (or ``h``) says where they go.  Gradients are not passed
    on: 8-bit matrices are constants to autograd, and a new tensor made from elements that need a
    gradient (x and residual of a norm, a bias, g) has an error for its backward pass.  With ``out``
    or ``h`` such elements are refused, unless under torch.no_grad().

    Recorded into a graph, calls of one handle share a workspace apart from that of calls made at
    once: replays of such graphs go one after another, on whatever stream.  The handle is one host
    thread's at a time, as the C interface asks for; the launches of a weight_grad, which share the
    workspace, follow one another whatever other threads call (autograd runs backward passes on
    threads of its own)."""

    def __init__(self, device: int = 0, ctx=None):
        if not torch.cuda.is_available():
            raise RuntimeError("no ROCm device visible: the 8-bit operators have no CPU path")
        if ctx is not None and ctx.device != device:
            raise ValueError(f"the context's device is {ctx.device}, not {device}")
        self.dev = torch.device("cuda", device)
        torch.cuda.set_device(self.dev)
        self.own = ctx is None
        self.ctx = ctx or S.shifter_create(device, torch.cuda.current_stream(self.dev).cuda_stream)
        self.stream = self.ctx.stream
        self.work = None
        self.recorded = []                 # workspaces of recorded calls, which use them at every replay
        self._calls = load_calls()

    def close(self):
        if self.own and self.ctx is not None:
            S.shifter_destroy(self.ctx)
        self.ctx = None

    def _enter(self):
        """New tensors belong to torch's current stream; the kernels run on the handle's."""
        if _raw_stream(self.dev.index) != self.stream:
            raise RuntimeError("this handle runs on the stream it (or its context) was made on: make one under the other stream")
        return self.ctx.handle.value, self.dev.index

    def _room(self, need: int) -> torch.Tensor:
        """A workspace of `need` bytes at least, kept from call to call; recorded calls have their own."""
        recording = torch.cuda.is_current_stream_capturing()
        work = (self.recorded[-1] if self.recorded else None) if recording else self.work
        if work is None or work.numel() < need:            # what is returned is this call's, whatever other threads leave here
            work = torch.empty(need, dtype=torch.uint8, device=self.dev)
            if recording:
                self.recorded.append(work)
            else:
                self.work = work
        return work

    # ---- the operators --------------------------------------------------------------
    def quantize(self, x: torch.Tensor, relu: bool = False, out: Optional[Q8Matrix] = None) -> Q8Matrix:
        """Each row of x (relu: of its ReLU) by itself: scale = max |x| / 127, codes the nearest
        whole numbers of 127 x / max |x|.  A linear tensor's rows are its output channels."""
        return self._calls.quantize(*self._enter(), x, relu, out)

    def dequantize(self, m: Q8Matrix, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None):
        """code * scale in the element type (that of ``out`` where it is given)."""
        return self._calls.dequantize(*self._enter(), m, dtype, out)

    def rms_norm(self, x: torch.Tensor, weight: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None,
                 h: Optional[torch.Tensor] = None, out: Optional[Q8Matrix] = None):
        """(8-bit matrix of h * weight / sqrt(mean(h^2) + eps), h) with h = x + residual in x's
        type, or x itself without a residual.  h may be x or residual: then it is updated in place."""
        return self._calls.rms_norm(*self._enter(), x, weight, eps, residual, h, out)

    def matmul(self, a: Q8Matrix, b: Q8Matrix, bias: Optional[torch.Tensor] = None, relu: bool = False,
               dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """a times b transposed (b: a linear layer's weights), + bias, ReLU: [a.rows, b.rows]."""
        return self._calls.matmul(*self._enter(), a, b, bias, relu, dtype, out)

    def weight_grad(self, g: torch.Tensor, x: Q8Matrix, mask: Optional[torch.Tensor] = None,
                    out: Optional[torch.Tensor] = None, accumulate: bool = False) -> torch.Tensor:
        """g transposed times the values of x: the fp32 gradient [g's columns, x.cols] of a linear
        layer's weights.  mask: uint8, what of the gradient is kept (as apply_mask writes it);
        accumulate: added to ``out``.  Up to SHIFTER_Q8_MAX_SUM rows a call."""
        return self._calls.weight_grad(*self._enter(), g, x, mask, torch.float32, out, accumulate, self._room)


def _rows(x: torch.Tensor) -> torch.Tensor:
    """x with its columns side by side and its rows one after another."""
    return x if (x.shape[1] < 2 or x.stride(1) == 1) and (x.shape[0] < 2 or x.stride(0) >= x.shape[1]) else x.contiguous()


def _weight_grad(g: torch.Tensor, ops: Q8, x: Q8Matrix, mask: Optional[torch.Tensor]) -> torch.Tensor:
    most, dw = S.SHIFTER_Q8_MAX_SUM, None
    if x.rows <= most:
        return ops.weight_grad(g, x, mask=mask)
    for i in range(0, x.rows, most):           # as many rows as a sum holds, the next ones added
        dw = ops.weight_grad(g[i:i + most], Q8Matrix(x.q[i:i + most], x.scale[i:i + most], x.cols), mask=mask, out=dw,
                             accumulate=dw is not None)
    return dw


class _WeightGrad(torch.autograd.Function):
    """The weights' gradient where it may be differentiated again: an error then.  `link` ties the result to the layer,
    so that the way from it to the layer's operands leads through here."""
    @staticmethod
    def forward(ctx, g, link, ops, x, mask):
        return _weight_grad(g, ops, x, mask)

    @staticmethod
    def backward(ctx, v):
        raise RuntimeError("checkpointed_linear: the weights' gradient has no derivative of its own")


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, ops, mask):
        kept = ops.quantize(_rows(x))
        link = x.new_empty(0)
        ctx.save_for_backward(kept.q, kept.scale, weight, link, *(() if mask is None else (mask,)))
        ctx.ops, ctx.cols = ops, kept.cols
        ctx.set_materialize_grads(False)
        return x @ weight.t(), link

    @staticmethod
    def backward(ctx, g, _):
        if g is None:
            return None, None, None, None
        q, scale, weight, link, *mask = ctx.saved_tensors
        g = _rows(g)
        # under autocast the product had the type that g has
        dx = g @ weight.to(g.dtype) if ctx.needs_input_grad[0] else None
        dw = None
        if ctx.needs_input_grad[1]:
            operands = ctx.ops, Q8Matrix(q, scale, ctx.cols), mask[0] if mask else None
            dw = _WeightGrad.apply(g, link, *operands) if torch.is_grad_enabled() else _weight_grad(g, *operands)
            dw = dw.to(weight.dtype)
        return dx, dw, None, None


def checkpointed_linear(x: torch.Tensor, weight: torch.Tensor, ops: Q8, mask: Optional[torch.Tensor] = None):
    """x [..., in] times weight [out, in] transposed, keeping x for the backward pass in 8 bits (a
    quarter of its fp32 size): the product and x's gradient are torch's, the weights' gradient comes
    from the 8-bit rows.  mask: uint8 [out, in], weights that were pruned get no gradient.  The
    weights' gradient can not be differentiated again, which is an error; x's can."""
    if mask is not None:
        if mask.dtype != torch.uint8 or mask.shape != weight.shape or mask.device != weight.device:
            raise ValueError("mask must be uint8, of the weights' shape and on their device")
        mask = _rows(mask)
    if x.dim() == 2:
        return _Linear.apply(x, weight, ops, mask)[0]
    rows = x.reshape(x.shape[:-1].numel(), x.shape[-1])
    return _Linear.apply(rows, weight, ops, mask)[0].view(*x.shape[:-1], weight.shape[0])
