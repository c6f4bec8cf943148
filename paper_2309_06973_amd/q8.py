"""8-bit matrices next to the prune-and-compact pass: a rebuilt variant's linear layers served
in 8 bits, and 8-bit activations kept for the backward pass while a masked network trains on.  Beside
them, what such a network is trained on and answers with: log probabilities and their gradient, the norm of
all gradients and their clipping, and low-rank adapters of many requests with their gradients.

Every step runs in libshifter's HIP kernels on the stream that was current when the handle (or
the context that it was given) was made; a call's checks, its new tensors and the way into the C ABI are _q8.so's (csrc/q8_bind.cpp).
Raises if no ROCm device is visible."""
from __future__ import annotations

import importlib.machinery
import importlib.util
import os
from typing import NamedTuple, Optional

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


class LogProbs(NamedTuple):
    """What Q8.log_probs returns; None for what was not asked for."""
    logp: Optional[torch.Tensor]           # [rows] of the targets
    lse: torch.Tensor                      # [rows] log sum exp
    entropy: Optional[torch.Tensor]        # [rows]
    top: Optional[torch.Tensor]            # [rows, top] log probabilities, largest first
    index: Optional[torch.Tensor]          # [rows, top] their columns
    norm: torch.Tensor                     # [rows, 2] what log_probs_grad works from: max x, log sum exp (z - scale max x)


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
    """The 8-bit operators and those beside them on one device and stream: the current one, or those of a given context.
    Matrices of elements are two-dimensional fp32, bf16 or fp16 tensors whose columns lie side by
    side; their rows may have any stride.
    Results are new tensors unless ``out`` (or ``h``) says where they go.  Gradients are not passed
    on: 8-bit matrices are constants to autograd, and a new tensor made from elements that need a
    gradient (x and residual of a norm, a bias, g) has an error for its backward pass.  With ``out``
    or ``h`` such elements are refused, unless under torch.no_grad().  The module's functions do pass gradients on.

    Recorded into a graph, calls of one handle share a workspace apart from that of calls made at
    once: replays of such graphs go one after another, on whatever stream.  The handle is one host
    thread's at a time, as the C interface asks for; the launches of a call that has several, which share a
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
        self.joined, self.recorded_joined = None, []       # the same for calls whose blocks join their sums: they start with zeros
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

    def _joined(self, need: int) -> torch.Tensor:
        """The same for the calls that find zeros at its front and leave zeros there: none else may write it."""
        recording = torch.cuda.is_current_stream_capturing()
        work = (self.recorded_joined[-1] if self.recorded_joined else None) if recording else self.joined
        new = work is None or work.numel() < need
        if new:
            with torch.inference_mode(False):      # or only calls in that mode could write it
                work = torch.empty(need, dtype=torch.uint8, device=self.dev)
            if recording:
                self.recorded_joined.append(work)
            else:
                self.joined = work
        if new or recording:           # recorded with each call: what a capture records is not done, and any graph may be replayed first
            work[:S.SHIFTER_LEARN_ZERO].zero_()
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

    def log_probs(self, x: torch.Tensor, target: Optional[torch.Tensor] = None, scale: float = 1.0, entropy: bool = False,
                  top: int = 0) -> LogProbs:
        """Of each row z = scale * x: log sum exp z, the log probability of column target[row] (int64; 0 where
        it is negative, NaN where it is not below the columns), the entropy, and the ``top`` largest log
        probabilities (up to SHIFTER_LOG_PROBS_MAX_TOP; equal logits: the lower column first) with their columns.  All
        numbers are fp32.  Minus infinity has probability 0; a row with NaN or infinity is NaN.  scale: above 0, up to 2^64."""
        return LogProbs(*self._calls.log_probs(*self._enter(), x, target, scale, entropy, top, self._joined))

    def log_probs_grad(self, x: torch.Tensor, target: Optional[torch.Tensor], norm: torch.Tensor,
                       g_logp: Optional[torch.Tensor] = None, g_lse: Optional[torch.Tensor] = None,
                       entropy: Optional[torch.Tensor] = None, g_entropy: Optional[torch.Tensor] = None, scale: float = 1.0,
                       out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x's gradient in x's type, from the gradients of log_probs' results (fp32 vectors, None: none); norm, and
        entropy with g_entropy, as log_probs gave them.  ``out`` may be x."""
        return self._calls.log_probs_grad(*self._enter(), x, target, norm, g_logp, g_lse, entropy, g_entropy, scale, out)

    def grad_norm(self, grads, masks=None) -> torch.Tensor:
        """The norm of all elements of a list of tensors (fp32, bf16, fp16, mixed as they come; any shape and dense layout), a
        0-dimensional fp32 tensor worked out in 64 bits.  masks: a list of uint8 tensors or None, laid out as
        their gradients: what is kept of each (as apply_mask writes them)."""
        return self._calls.grad_norm(*self._enter(), grads, masks, None, None, self._joined)

    def clip_grad_norm(self, grads, max_norm: float, masks=None, out=None) -> torch.Tensor:
        """The same norm, and the gradients times min(1, max_norm / (norm + 1e-6)), masked elements 0, written in place or to
        the tensors of ``out`` (laid out as their gradients).  What is written may not overlap anything else."""
        return self._calls.grad_norm(*self._enter(), grads, masks, float(max_norm), out, self._joined)

    def adapters(self, y: torch.Tensor, x, a: torch.Tensor, b: torch.Tensor, which: torch.Tensor,
                 scale: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                 down: Optional[torch.Tensor] = None) -> torch.Tensor:
        """y + scale[i] * (x a[i]') b[i]' for each row, i = which[row] (int64; negative: no adapter, not below the adapters:
        NaN): low-rank adapters of many requests beside a projection that gave y.  x: elements of a's type, or the
        Q8Matrix that the projection read.  a: [adapters, rank, x's columns], b: [adapters, y's columns, rank], rank up to
        SHIFTER_ADAPTERS_MAX_RANK.  ``out`` may be y; down: fp32 [rows, rank], gets scale[i] * x a[i]' for adapters_grad."""
        return self._calls.adapters(*self._enter(), y, x, a, b, which, scale, out, down, self._room)

    def adapters_grad(self, g: torch.Tensor, x, a: torch.Tensor, b: torch.Tensor, which: torch.Tensor,
                      scale: Optional[torch.Tensor] = None, down: Optional[torch.Tensor] = None, dx: bool = True):
        """(gradient of x in a's type or None, of a and of b in fp32) from g, that of adapters' result, in a's type; y's is g
        itself.  down: as adapters wrote it, or it is worked out again."""
        return self._calls.adapters_grad(*self._enter(), g, x, a, b, which, scale, down, dx, self._room)


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


def _recording(what: str, *tensors: torch.Tensor):
    """A backward pass is recorded by recording the gradient's own call."""
    if torch.cuda.is_current_stream_capturing() and torch.is_grad_enabled() and any(t.requires_grad for t in tensors):
        raise RuntimeError(f"{what} can not be recorded where a gradient is needed: record the handle's calls, the gradient's too")


class _LogProbsGrad(torch.autograd.Function):
    """x's gradient where it may be differentiated again: an error then."""
    @staticmethod
    def forward(ctx, x, g_logp, g_entropy, g_lse, ops, target, norm, entropy, scale):
        return ops.log_probs_grad(x, target, norm, g_logp, g_lse, entropy, g_entropy, scale)

    @staticmethod
    def backward(ctx, v):
        raise RuntimeError("target_log_probs: x's gradient has no derivative of its own")


class _LogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, target, ops, scale):
        r = ops.log_probs(x, target, scale=scale, entropy=True)
        ctx.save_for_backward(x, target, r.norm, r.entropy)
        ctx.ops, ctx.scale = ops, scale
        ctx.set_materialize_grads(False)
        return r.logp, r.entropy, r.lse

    @staticmethod
    def backward(ctx, *grads):
        x, target, norm, entropy = ctx.saved_tensors
        if all(g is None for g in grads):
            return None, None, None, None
        g_logp, g_entropy, g_lse = (None if g is None else g.contiguous() for g in grads)
        dx = _LogProbsGrad.apply(x, g_logp, g_entropy, g_lse, ctx.ops, target, norm, entropy.detach(), ctx.scale)
        return dx, None, None, None


def target_log_probs(x: torch.Tensor, target: torch.Tensor, ops: Q8, scale: float = 1.0):
    """(log probabilities of the targets, entropies, log sum exp) of the rows of scale * x [..., columns], fp32 [...]:
    Q8.log_probs with its gradient.  target: int64 [...], negative: left out (0, without gradient).  The gradient can
    not be differentiated again, which is an error, and not be recorded: log_probs and log_probs_grad can."""
    if target.shape != x.shape[:-1]:
        raise ValueError("target must have x's shape without its last dimension")
    _recording("target_log_probs", x)
    rows = _rows(x.reshape(target.numel(), x.shape[-1]))
    return tuple(t.view(target.shape) for t in _LogProbs.apply(rows, target.reshape(-1).contiguous(), ops, scale))


class _AdaptersGrad(torch.autograd.Function):
    """The gradients where they may be differentiated again: an error then."""
    @staticmethod
    def forward(ctx, g, x, a, b, ops, x8, which, scale, down, dx):
        got = ops.adapters_grad(g, x if x8 is None else x8, a, b, which, scale, down, dx)
        return got if got[0] is not None else (got[1].new_empty(0), *got[1:])

    @staticmethod
    def backward(ctx, *v):
        raise RuntimeError("adapted: the gradients have no derivative of their own")


class _Adapted(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, x, a, b, ops, x8, which, scale):
        down = torch.empty(y.shape[0], a.shape[1], dtype=torch.float32, device=y.device)
        out = ops.adapters(y, x if x8 is None else x8, a, b, which, scale, down=down)
        ctx.save_for_backward(x, a, b, which, down, *(t for t in (scale, *((x8.q, x8.scale) if x8 is not None else ())) if t is not None))
        ctx.ops, ctx.scaled, ctx.cols = ops, scale is not None, None if x8 is None else x8.cols
        return out

    @staticmethod
    def backward(ctx, g):
        x, a, b, which, down, *rest = ctx.saved_tensors
        scale = rest.pop(0) if ctx.scaled else None
        x8 = Q8Matrix(*rest, ctx.cols) if rest else None
        dx = da = db = None
        if any(ctx.needs_input_grad[1:4]):
            dx, da, db = _AdaptersGrad.apply(_rows(g), x, a, b, ctx.ops, x8, which, scale, down, ctx.needs_input_grad[1])
            dx = dx if ctx.needs_input_grad[1] else None
            da, db = da.to(a.dtype), db.to(b.dtype)
        return g, dx, da, db, None, None, None, None


def adapted(y: torch.Tensor, x, a: torch.Tensor, b: torch.Tensor, which: torch.Tensor, ops: Q8,
            scale: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Q8.adapters with the gradients of y, x (unless it is a Q8Matrix), a and b: y and x [..., columns] of a's type,
    which int64 [...].  scale is a constant.  The gradients can not be differentiated again, which is an error, and not be
    recorded: adapters and adapters_grad can."""
    if scale is not None and scale.requires_grad and torch.is_grad_enabled():
        raise ValueError("scale needs a gradient, which adapted does not pass on: detach it")
    if y.dtype != a.dtype:
        raise ValueError("y must have the adapters' type")
    x8 = x if isinstance(x, Q8Matrix) else None
    if which.shape != y.shape[:-1] or (x8 is None and x.shape[:-1] != which.shape):
        raise ValueError("which must have y's and x's shape without their last dimension")
    _recording("adapted", y, a, b, *(() if x8 is not None else (x,)))
    flat = y.new_empty(0) if x8 is not None else _rows(x.reshape(which.numel(), x.shape[-1]))
    out = _Adapted.apply(_rows(y.reshape(which.numel(), y.shape[-1])), flat, a.contiguous(), b.contiguous(), ops, x8,
                         which.reshape(-1).contiguous(), scale)
    return out.view(y.shape)
