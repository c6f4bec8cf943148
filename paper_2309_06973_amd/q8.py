"""8-bit matrices next to the prune-and-compact pass: a rebuilt variant's linear layers served
in 8 bits, and 8-bit activations kept for the backward pass while a masked network trains on.

Buffer management and argument marshalling only: every step runs in libshifter's HIP kernels
on the stream that was current when the handle was made.  Raises if no ROCm device is visible."""
from __future__ import annotations

from typing import Optional

import torch

from . import shifter as S

_DTYPES = {torch.float32: S.SHIFTER_F32, torch.bfloat16: S.SHIFTER_BF16, torch.float16: S.SHIFTER_F16}
# a call's kernel takes a few microseconds: the checks around it are kept short (the stream object of
# torch.cuda.current_stream alone costs 1.9 us, this 0.1)
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None


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


class Q8:
    """The 8-bit operators on one device and stream.  Matrices of elements are two-dimensional
    fp32, bf16 or fp16 tensors whose columns lie side by side; their rows may have any stride.
    Results are new tensors unless ``out`` (or ``h``) says where they go."""

    def __init__(self, device: int = 0, ctx=None):
        if not torch.cuda.is_available():
            raise RuntimeError("no ROCm device visible: the 8-bit operators have no CPU path")
        self.dev = torch.device("cuda", device)
        torch.cuda.set_device(self.dev)
        self.stream = torch.cuda.current_stream(self.dev).cuda_stream
        self.own = ctx is None
        self.ctx = ctx or S.shifter_create(device, self.stream)
        self.work = None
        self.recorded = []                 # workspaces that a recorded call holds
        self._int8 = torch.empty(0, dtype=torch.int8, device=self.dev)        # new_empty is the shortest way to a new tensor
        self._float = torch.empty(0, dtype=torch.float32, device=self.dev)

    def close(self):
        if self.own and self.ctx is not None:
            S.shifter_destroy(self.ctx)
        self.ctx = None

    # ---- checks -------------------------------------------------------------------
    def _enter(self):
        """New tensors belong to torch's current stream; the kernels run on the handle's."""
        if _raw_stream(self.dev.index) != self.stream:
            raise RuntimeError("this handle runs on the stream it was made on: make one under the other stream")

    def _matrix(self, x: torch.Tensor, what: str):
        """(dtype code, rows, cols, stride)"""
        code = _DTYPES.get(x.dtype)
        if code is None or x.dim() != 2:
            raise ValueError(f"{what} must be a two-dimensional fp32, bf16 or fp16 tensor")
        rows, cols = x.shape
        ld, side = x.stride()
        if rows < 2:
            ld = cols
        if (cols > 1 and side != 1) or ld < cols:
            raise ValueError(f"the columns of {what} must lie side by side, rows one after another")
        self._here(x, what)
        return code, rows, cols, ld

    def _here(self, x: torch.Tensor, what: str):
        if x.device != self.dev:
            raise ValueError(f"{what} is not on {self.dev}")

    def _vector(self, v: torch.Tensor, n: int, what: str):
        if v.dtype != torch.float32 or v.shape != (n,) or not v.is_contiguous():
            raise ValueError(f"{what} must be a contiguous float32 vector of {n}")
        self._here(v, what)

    def _same(self, a: torch.Tensor, shape, dtype, what: str):
        if a.shape != shape or a.dtype != dtype:
            raise ValueError(f"{what} must have shape {tuple(shape)} and type {dtype}")

    def _room(self, rows: int, cols: int, out: Optional[Q8Matrix]) -> Q8Matrix:
        if out is None:
            m = Q8Matrix.__new__(Q8Matrix)             # as __init__ would leave it
            m.rows, m.cols, m.ld = rows, cols, _pad(cols)
            m.q = self._int8.new_empty(rows, m.ld)
            m.scale = self._float.new_empty(rows)
            return m
        self._here(out.q, "out")
        if out.rows != rows or out.cols != cols:
            raise ValueError("out is an 8-bit matrix of another size")
        return out

    def _result(self, rows: int, cols: int, dtype: torch.dtype, out: Optional[torch.Tensor]):
        """(out or a new matrix, dtype code, stride)"""
        if out is None:
            code = _DTYPES.get(dtype)
            if code is None:
                raise ValueError("dtype must be fp32, bf16 or fp16")
            return torch.empty((rows, cols), dtype=dtype, device=self.dev), code, cols
        code, _, _, ld = self._matrix(out, "out")
        self._same(out, (rows, cols), out.dtype, "out")
        return out, code, ld

    # ---- the operators --------------------------------------------------------------
    def quantize(self, x: torch.Tensor, relu: bool = False, out: Optional[Q8Matrix] = None) -> Q8Matrix:
        """Each row of x (relu: of its ReLU) by itself: scale = max |x| / 127, codes the nearest
        whole numbers of 127 x / max |x|.  A linear tensor's rows are its output channels."""
        self._enter()
        t, rows, cols, ld = self._matrix(x, "x")
        m = self._room(rows, cols, out)
        S.shifter_quantize_q8(self.ctx, x, t, ld, rows, cols, S.SHIFTER_Q8_RELU if relu else 0, m.q, m.ld, m.scale)
        return m

    def dequantize(self, m: Q8Matrix, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None):
        """code * scale in the element type (that of ``out`` where it is given)."""
        self._enter()
        self._here(m.q, "m")
        out, t, ld = self._result(m.rows, m.cols, dtype, out)
        S.shifter_dequantize_q8(self.ctx, m.q, m.ld, m.scale, m.rows, m.cols, out, t, ld)
        return out

    def rms_norm(self, x: torch.Tensor, weight: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None,
                 h: Optional[torch.Tensor] = None, out: Optional[Q8Matrix] = None):
        """(8-bit matrix of h * weight / sqrt(mean(h^2) + eps), h) with h = x + residual in x's
        type, or x itself without a residual.  h may be x or residual: then it is updated in place."""
        self._enter()
        t, rows, cols, ld = self._matrix(x, "x")
        self._vector(weight, cols, "weight")
        ld_r = ld_h = 0
        if residual is not None:
            self._same(residual, x.shape, x.dtype, "residual")
            _, _, _, ld_r = self._matrix(residual, "residual")
            if h is None:
                h, ld_h = x.new_empty(rows, cols), cols
            else:
                self._same(h, x.shape, x.dtype, "h")
                _, _, _, ld_h = self._matrix(h, "h")
        elif h is not None:
            raise ValueError("h without a residual: the stream is x itself")
        m = self._room(rows, cols, out)
        S.shifter_rms_norm_q8(self.ctx, x, ld, residual, ld_r, t, rows, cols, weight, eps, h, ld_h, m.q, m.ld, m.scale)
        return m, x if h is None else h

    def matmul(self, a: Q8Matrix, b: Q8Matrix, bias: Optional[torch.Tensor] = None, relu: bool = False,
               dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """a times b transposed (b: a linear layer's weights), + bias, ReLU: [a.rows, b.rows]."""
        self._enter()
        self._here(a.q, "a")
        self._here(b.q, "b")
        if a.cols != b.cols:
            raise ValueError("a and b have different numbers of columns")
        if bias is not None:
            self._vector(bias, b.rows, "bias")
        out, t, ld = self._result(a.rows, b.rows, dtype, out)
        S.shifter_matmul_q8(self.ctx, a.q, a.ld, a.scale, b.q, b.ld, b.scale, a.rows, b.rows, a.cols, bias,
                            S.SHIFTER_Q8_RELU if relu else 0, out, t, ld)
        return out

    def weight_grad(self, g: torch.Tensor, x: Q8Matrix, mask: Optional[torch.Tensor] = None,
                    out: Optional[torch.Tensor] = None, accumulate: bool = False) -> torch.Tensor:
        """g transposed times the values of x: the fp32 gradient [g's columns, x.cols] of a linear
        layer's weights.  mask: uint8, what of the gradient is kept (as apply_mask writes it);
        accumulate: added to ``out``."""
        self._enter()
        t, m, n, ld = self._matrix(g, "g")
        self._here(x.q, "x")
        if x.rows != m:
            raise ValueError("g and x have different numbers of rows")
        k, ld_mask = x.cols, 0
        if mask is not None:
            self._same(mask, (n, k), torch.uint8, "mask")
            self._here(mask, "mask")
            ld_mask = mask.stride(0) if n > 1 else k
            if (k > 1 and mask.stride(1) != 1) or ld_mask < k:
                raise ValueError("the columns of mask must lie side by side, rows one after another")
        if accumulate and out is None:
            raise ValueError("accumulate without out")
        if out is not None and out.dtype != torch.float32:
            raise ValueError("out must be float32")
        out, _, ld_out = self._result(n, k, torch.float32, out)
        need = S.shifter_weight_grad_q8_layout(m, n, k)
        work = None
        if need:
            if self.work is None or self.work.numel() < need:
                self.work = torch.empty(need, dtype=torch.uint8, device=self.dev)
            work = self.work
            if torch.cuda.is_current_stream_capturing() and not any(w is work for w in self.recorded):
                self.recorded.append(work)
        S.shifter_weight_grad_q8(self.ctx, g, t, ld, x.q, x.ld, x.scale, m, n, k, mask, ld_mask,
                                 S.SHIFTER_Q8_ACCUMULATE if accumulate else 0, out, ld_out, work, need)
        return out


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, ops, mask):
        kept = ops.quantize(x)
        ctx.save_for_backward(kept.q, kept.scale, weight, *(() if mask is None else (mask,)))
        ctx.ops, ctx.cols = ops, kept.cols
        return x @ weight.t()

    @staticmethod
    def backward(ctx, g):
        q, scale, weight, *mask = ctx.saved_tensors
        g = g if g.dim() == 2 and (g.shape[1] < 2 or g.stride(1) == 1) and (g.shape[0] < 2 or g.stride(0) >= g.shape[1]) \
            else g.contiguous()
        dx = g @ weight if ctx.needs_input_grad[0] else None
        dw = None
        if ctx.needs_input_grad[1]:
            dw = ctx.ops.weight_grad(g, Q8Matrix(q, scale, ctx.cols), mask=mask[0] if mask else None).to(weight.dtype)
        return dx, dw, None, None


def checkpointed_linear(x: torch.Tensor, weight: torch.Tensor, ops: Q8, mask: Optional[torch.Tensor] = None):
    """x times weight transposed, keeping x for the backward pass in 8 bits (a quarter of its fp32
    size): the product and x's gradient are torch's, the weights' gradient comes from the 8-bit
    rows.  mask: uint8 [out, in], weights that were pruned get no gradient."""
    return _Linear.apply(x, weight, ops, mask)
