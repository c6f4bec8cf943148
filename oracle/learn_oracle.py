"""Log probabilities, gradient norms and adapters from their definitions, in 64 bits on the CPU (test infrastructure
only), with how far a kernel that works in 32 bits may be from them."""
import numpy as np
import torch

U = 2.0 ** -24                       # half a step of fp32, relative
HALF_STEP = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
# half the smallest step there is, for results below the normal numbers
LEAST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


class Logs:
    """Rows of logits x (elements, any device): lse, p, entropy in float64, and bounds of a 32-bit kernel's errors.

    A kernel sums e = 2^d, d = (x - m) c, c = scale log2 e.  d has three roundings (x - m, c, the product), so e is off by
    3 U |z - m| + 2 U (2^d itself: one unit in the last place), relatively.  Each time a thread's largest grows its sums take one
    more such factor; those steps of d add up to no more than |z - m| of the terms before, so a term takes the
    roundings of its d twice over, and 3 U for each step.  `adds` bounds additions and steps on a term's way.  Weighted with p that is
        rel(s) <= U (6 D + 4 adds + 8),   D = sum p |z - m|
        off(u / s) <= U (6 E + D (4 adds + 8)) + D rel(s),   E = sum p (z - m)^2
    and log s is off by rel(s), lse and log p by that and their own rounding, H by both."""

    def __init__(self, x, scale=1.0):
        self.x = x.detach().cpu().double().numpy()
        self.scale = float(np.float32(scale))
        z = self.x * self.scale
        rows, cols = z.shape
        with np.errstate(all="ignore"):
            m = z.max(axis=1, keepdims=True, initial=-np.inf)
            at = np.where(np.isfinite(m), m, 0.0)
            e = np.exp(z - at)
            s = e.sum(axis=1, keepdims=True)
            self.lse = (at + np.log(s))[:, 0]
            self.lse[np.isnan(z).any(axis=1) | (m[:, 0] == np.inf)] = np.nan
            self.log_s = np.log(s)[:, 0]
            self.log_s[np.isnan(self.lse)] = np.nan
            self.norm = np.stack([np.where(np.isneginf(m[:, 0]), np.finfo(np.float32).min, m[:, 0] / self.scale), self.log_s], 1)
            self.log_p = z - at - self.log_s[:, None]
            self.p = np.exp(self.log_p)
            terms = np.where(self.p == 0, 0.0, self.p * self.log_p)
            self.entropy = -terms.sum(axis=1)
            self.entropy[~np.isfinite(self.lse)] = np.nan
            d = np.where(self.p == 0, 0.0, z - at)
            big_d, big_e = (self.p * np.abs(d)).sum(axis=1), (self.p * d * d).sum(axis=1)
        threads = 16 if cols <= 256 else 64 if cols <= 1024 else 256
        adds = cols / threads + 24
        self.rel = U * (6 * big_d + 4 * adds + 8)
        self.off_h = self.rel + U * (6 * big_e + big_d * (4 * adds + 8)) + big_d * self.rel

    def logp(self, target):
        t = target.cpu().numpy()
        cols = self.x.shape[1]
        got = np.array([self.log_p[r, c] if 0 <= c < cols else (0.0 if c < 0 else np.nan) for r, c in enumerate(t)])
        return got

    def top(self, k):
        """Columns of the k largest logits, equal ones in order; NaN with minus infinity."""
        key = np.where(np.isnan(self.x), -np.inf, self.x)
        return np.argsort(-key, axis=1, kind="stable")[:, :k]

    def grad(self, target, g_logp=None, g_lse=None, g_entropy=None):
        """(gradient in float64, how far a 32-bit kernel's may be before its rounding to x's type), given log s and
        entropy rounded to fp32.  d = fl(scale fl(x - m) - log s): U (2 |z - m| + |log s| + |d|) <= U (3 |d| + 3 |log s|); p: that, 2
        roundings of d log2 e, 2 U of 2^d."""
        rows, cols = self.x.shape
        v = lambda g: np.zeros(rows) if g is None else g.detach().cpu().double().numpy()
        t = target.cpu().numpy() if target is not None else np.full(rows, -1)
        one, of_lse, of_h = np.where(t >= 0, v(g_logp), 0.0), v(g_lse), v(g_entropy)
        with np.errstate(all="ignore"):
            log_p = np.where(self.p == 0, 0.0, self.log_p)
            h = np.where(of_h == 0, 0.0, self.entropy)[:, None]
            factor = (of_lse - one)[:, None] - of_h[:, None] * (log_p + h)
            size = np.abs(of_lse)[:, None] + np.abs(one)[:, None] + np.abs(of_h[:, None]) * (np.abs(log_p) + np.abs(h))
            want = self.p * factor
            off_d = U * (3 * np.abs(self.log_s)[:, None] + 3 * np.abs(log_p))
            off = self.p * (size * (off_d + U * (2 * np.abs(log_p) + 2) + 6 * U) + np.abs(of_h[:, None]) * (off_d + U * np.abs(h)))
        for r, c in enumerate(t):
            if 0 <= c < cols:
                want[r, c] += one[r]
                off[r, c] += 2 * U * (abs(one[r]) + abs(want[r, c]))
            elif c >= cols:
                want[r] = np.nan
        none = (one == 0) & (of_lse == 0) & (of_h == 0) & (t < cols)
        want[none] = 0.0
        off[none] = 0.0
        return want * self.scale, off * self.scale * (1 + 2 * U) + 2 * U * np.abs(want * self.scale)


def clipped(grads, max_norm, masks=None):
    """(norm, results) in float64."""
    kept = [g.detach().cpu().double() if masks is None or masks[i] is None else
            torch.where(masks[i].cpu() != 0, g.detach().cpu().double(), 0.0) for i, g in enumerate(grads)]
    norm = float(torch.sqrt(sum((k * k).sum() for k in kept) + torch.zeros((), dtype=torch.float64)))
    by = max_norm / (norm + 1e-6)
    factor = 1.0 if by >= 1.0 else by              # NaN stays
    return norm, [torch.where(k == 0, k, k * factor) if np.isfinite(factor) else
                  (k * factor if masks is None or masks[i] is None else torch.where(masks[i].cpu() != 0, k * factor, 0.0))
                  for i, k in enumerate(kept)]


class Adapters:
    """out = y + scale[i] (x a[i]') b[i]' and its gradients in float64 on the CPU, and how far a kernel may be that sums in 32
    bits: a sum of n products is off by 2 U (n + 40) of the sum of their sizes at most (products of 16-bit factors are exact,
    others off by U; every addition may cut instead of round; parts and wavefronts are joined in no more than 40 further
    ones; the scales cost 2 U).  An intermediate's error goes on with the sizes of what it is multiplied with."""

    def __init__(self, y, x, a, b, which, scale=None):
        d = lambda t: t.detach().cpu().double()
        self.y, self.x, self.a, self.b = d(y), d(x), d(a), d(b)
        self.which = which.cpu()
        many = self.a.shape[0]
        self.scale = d(scale) if scale is not None else torch.ones(many, dtype=torch.float64)
        self.many = many
        rank = self.a.shape[1]
        self.down, self.off_down = torch.zeros(len(self.which), rank, dtype=torch.float64), torch.zeros(len(self.which), rank, dtype=torch.float64)
        self.out, self.off = self.y.clone(), torch.zeros_like(self.y)
        err = lambda n: 2 * U * (n + 40)
        k = self.a.shape[2]
        for i, rows in self.rows():
            c, a_, b_ = abs(self.scale[i]), self.a[i], self.b[i]
            self.down[rows] = self.scale[i] * (self.x[rows] @ a_.t())
            self.off_down[rows] = err(k) * c * (self.x[rows].abs() @ a_.abs().t())
            part = self.down[rows] @ b_.t()
            self.out[rows] += part
            self.off[rows] = self.off_down[rows] @ b_.abs().t() + err(rank) * (self.down[rows].abs() @ b_.abs().t()) + U * self.out[rows].abs()
        bad = self.which >= many
        self.out[bad], self.down[bad] = float("nan"), float("nan")

    def rows(self):
        for i in range(self.many):
            rows = torch.nonzero(self.which == i)[:, 0]
            if len(rows):
                yield i, rows

    def grads(self, g):
        """{name: (gradient, bound)}."""
        g = g.detach().cpu().double()
        err = lambda n: 2 * U * (n + 40)
        zero = lambda t: torch.zeros(t.shape, dtype=torch.float64)
        dx, dx_off, da, da_off, db, db_off = (zero(t) for t in (self.x, self.x, self.a, self.a, self.b, self.b))
        n, rank = self.b.shape[1:]
        for i, rows in self.rows():
            c, a, b, x = abs(self.scale[i]), self.a[i], self.b[i], self.x[rows]
            up = self.scale[i] * (g[rows] @ b)
            up_off = err(n) * c * (g[rows].abs() @ b.abs())
            dx[rows] = up @ a
            dx_off[rows] = up_off @ a.abs() + err(rank) * (up.abs() @ a.abs())
            da[i] = up.t() @ x
            da_off[i] = up_off.t() @ x.abs() + err(len(rows)) * (up.abs().t() @ x.abs())
            db[i] = g[rows].t() @ self.down[rows]
            db_off[i] = g[rows].abs().t() @ self.off_down[rows] + err(len(rows)) * (g[rows].abs().t() @ self.down[rows].abs())
        dx[self.which >= self.many] = float("nan")
        return dict(dx=(dx, dx_off), da=(da, da_off), db=(db, db_off))
