"""Plain 64-bit forms of the accumulated attention weights, the 8-bit cache and the eviction from it, for their
tests: written from the definitions in include/twinkv.h.  torch float64 tensors on any device."""
import math

import torch

U = 2.0 ** -24   # half a unit in the last place of fp32, relative
BLOCK = 32


def weights(q, k, lse, seen, scale):
    """One head: q (m, d), k (n, d) in float64, lse (m,), seen (m, n): the weights, and what fp32 arithmetic may be
    off by in each.  A score is a sum of d products, scaled and taken in units of log2 (d + 8 roundings of at most
    the sum of its magnitudes); the log-sum-exp is scaled too and the difference rounded (2 of each); and the
    exponential (2)."""
    s = (q @ k.T) * scale
    size = (q.abs() @ k.abs().T) * abs(scale)
    w = torch.exp(s - lse[:, None])
    off = w * ((q.shape[1] + 8) * size + 2 * lse.abs()[:, None] + 2 * s.abs() + 4) * U
    dead = ~seen | (lse == -math.inf)[:, None]
    return w.masked_fill(dead, 0.0), off.masked_fill(dead, 0.0)


def mass_of(q, k, lse, seen, scale, before=None):
    """q (G, m, d) and lse (G, m) of the query heads that share k (n, d): what each key receives, and the tolerance:
    the weights' own, and a rounding for every addition (over m G rows, in any order)."""
    total = torch.zeros(k.shape[0], dtype=torch.float64, device=k.device)
    tol = torch.zeros_like(total)
    for g in range(q.shape[0]):
        w, off = weights(q[g], k, lse[g], seen, scale)
        total, tol = total + w.sum(0), tol + off.sum(0)
    tol = tol + (q.shape[0] * q.shape[1] + 8) * U * total
    if before is not None:
        total = total + before
        tol = tol + U * total.abs()
    return total, tol + 1e-30


def byte_of(top):
    """The scale's byte for a block whose largest magnitude is top."""
    for b in range(1, 248):
        if top < 127.5 * 2.0 ** (b - 127):
            return b
    return 248


def on_grid(x, byte):
    """The values that float64 rows have on a block's grid (torch.round: ties to the even number)."""
    s = 2.0 ** (byte - 127)
    return torch.round(x / s).clamp(-127, 127) * s


class Rows8:
    """The keys (or values) of one problem as the cache holds them: their values and every block's byte."""

    def __init__(self, d, device):
        self.x = torch.zeros((0, d), dtype=torch.float64, device=device)
        self.bytes = []

    def append(self, new):
        """new (n, d) float64.  Returns whether a row was not finite."""
        finite = torch.isfinite(new).all(1)
        new = torch.where(finite[:, None], new, torch.zeros_like(new))
        done = 0
        while done < len(new):
            n = len(self.x)
            a, lo = n // BLOCK * BLOCK, n % BLOCK
            part = new[done:done + BLOCK - lo]
            byte = byte_of(float(part.abs().max()))
            if lo:
                byte = max(byte, self.bytes[-1])
                self.bytes[-1] = byte
            else:
                self.bytes.append(byte)
            self.x = torch.cat([self.x[:a], on_grid(self.x[a:], byte), on_grid(part, byte)])
            done += len(part)
        return not bool(finite.all())


def stored(x):
    """Rows as a compaction stores them, all at once."""
    r = Rows8(x.shape[1], x.device)
    bad = r.append(x)
    return r.x, r.bytes, bad


def kept_rows(mass, n, budget, n_sink, n_recent):
    """The rows of n that an eviction keeps, ascending; mass a list of Python floats."""
    def rank(t):
        if t < n_sink or t >= n - n_recent:
            return (0, 0.0, t)
        return (2, 0.0, t) if math.isnan(mass[t]) else (1, -mass[t], t)
    return sorted(sorted(range(n), key=rank)[:min(n, budget)])
