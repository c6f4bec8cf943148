"""The 8-bit operators from their definition, in 64 bits on the CPU (numpy; test infrastructure
only).  Rounded element types are torch's; everything else is float64 or whole numbers."""
import numpy as np
import torch

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
U32 = 2.0 ** -24                       # half a step of fp32, relative
TINY32 = 2.0 ** -149
HALF_STEP = {n: torch.finfo(t).eps / 2 for n, t in DTYPES.items()}
# half the smallest step there is, for results below the normal numbers
LEAST = {"fp32": 2.0 ** -150, "bf16": 2.0 ** -134, "fp16": 2.0 ** -25}


def f64(t):
    """A tensor of elements as float64 (exact)."""
    return t.detach().cpu().double().numpy()


def codes(p):
    """(codes, largest magnitude) of rows of float64 values that are 24-bit numbers."""
    p = np.asarray(p, dtype=np.float64)
    rows, cols = p.shape
    a = np.abs(p).max(axis=1, initial=0.0)
    fine = np.isfinite(p).all(axis=1)
    live = fine & (a > 0)
    q = np.zeros((rows, cols), dtype=np.int8)
    if cols and live.any():
        x, top = np.abs(p[live]), a[live][:, None]
        low = np.floor(127.0 * x / top)
        # next to a whole number the quotient may have been rounded up to it: bring it back
        low = np.where(127.0 * x < low * top, low - 1, low)
        rest = 254.0 * x - (2.0 * low + 1.0) * top            # exact: both are below 2^53 units
        up = (rest > 0) | ((rest == 0) & (low % 2 == 1))
        q[live] = (np.sign(p[live]) * (low + up)).astype(np.int8)
    return q, np.where(fine, a, np.nan)


def quantize(x, relu=False):
    """(codes, scales in 64 bits): scale NaN for a row that is not finite."""
    p = f64(x)
    if relu:
        p = np.where(p < 0, 0.0, p)
    q, a = codes(p)
    return q, a / 127.0


def rms_norm(x, weight, eps, residual=None):
    """(codes, scales in 64 bits, stream in x's type)."""
    h = x.detach().cpu()
    if residual is not None:
        h = (h.double() + residual.detach().cpu().double()).to(x.dtype)
    w = weight.detach().cpu().float().numpy()
    with np.errstate(over="ignore", invalid="ignore"):
        p = (h.float().numpy() * w).astype(np.float64)         # one fp32 rounding, by definition
        q, a = codes(p)
        h64 = f64(h)
        mean = (h64 ** 2).sum(axis=1) / max(1, h64.shape[1])
        scale = np.where(a == 0, 0.0, a / (127.0 * np.sqrt(np.where(a == 0, 1.0, mean + eps))))
    return q, scale, h


def product(qa, sa, qb, sb, bias=None, relu=False):
    """(result in 64 bits, its magnitude before the bias): whole-number sums, exact in float64."""
    s = qa.astype(np.float64) @ qb.astype(np.float64).T
    c = s * sa.astype(np.float64)[:, None] * sb.astype(np.float64)
    mag = np.abs(c)
    if bias is not None:
        c = c + bias.astype(np.float64)
    if relu:
        c = np.where(c < 0, 0.0, c)
    return c, mag


def weight_grad(g, q, s, mask=None):
    """(gradient in 64 bits, bound of the library's error before the roundings of what is added to)."""
    with np.errstate(invalid="ignore", over="ignore"):
        p = f64(g) * s.astype(np.float64)[:, None]
        q = q.astype(np.float64)
        d = p.T @ q
        top = np.abs(p).max(axis=0, initial=0.0)
        # a unit of the column's whole numbers a term, and the roundings of p, of the factor and its
        # inverse (2), of three conversions and sums, of the unit's product: 8 half steps of the terms
        bound = (top / 8355711.0)[:, None] * np.abs(q).sum(axis=0) + 8 * U32 * (np.abs(p).T @ np.abs(q)) + TINY32
    if mask is not None:
        d, bound = np.where(mask != 0, d, 0.0), np.where(mask != 0, bound, 0.0)
    return d, bound
