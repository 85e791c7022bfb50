"""Plain 64-bit forms of the operators around the cache, for their tests: written from the definitions
in include/twinkv.h, loops where loops say it best.  torch float64 tensors on any device."""
import math

import torch

U = 2.0 ** -24   # half a unit in the last place of fp32, relative
U16 = 2.0 ** -8  # of bf16 (8 significant bits where fp32 has 24)
GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def norm_rope(x, w, eps, rope, pos):
    """x (H, T, d) float64."""
    d = x.shape[-1]
    if w is not None:
        x = x * w.double() / ((x * x).sum(-1, keepdim=True) / d + eps).sqrt()
    if rope is None:
        return x
    p = pos.long()
    ok = (p >= 0) & (p < rope.shape[0])
    t = rope.double()[torch.where(ok, p, torch.zeros_like(p))]
    c, s = t[:, :d // 2], t[:, d // 2:]
    a, b = x[..., :d // 2], x[..., d // 2:]
    y = torch.cat([a * c - b * s, b * c + a * s], -1)
    y[:, ~ok] = math.nan
    return y


def seen_by(nq, nk, window, sink):
    """(nq, nk) which keys each query sees."""
    p = (nk - nq + torch.arange(nq))[:, None]
    j = torch.arange(nk)[None, :]
    return (j <= p) & ((p - j < window) | (j < sink))


def softmax_rows(q, k, v, seen, scale):
    """One head: q (m, d), k and v (n, d) in float64, seen (m, n).  Keys that a row does not see do not
    enter its sums.  Returns out, lse, sum of p |v|, and the largest scale * sum |q||k| a row sees."""
    m, d = q.shape
    out = torch.zeros((m, d), dtype=torch.float64, device=q.device)
    lse = torch.full((m,), -math.inf, dtype=torch.float64, device=q.device)
    mass = torch.zeros_like(out)
    size = torch.zeros((m,), dtype=torch.float64, device=q.device)
    for i in range(m):
        at = seen[i].nonzero().squeeze(1)
        if len(at) == 0:
            continue
        kk, vv = k[at], v[at]
        s = (kk @ q[i]) * scale
        lse[i] = torch.logsumexp(s, 0)
        p = torch.softmax(s, 0)
        out[i] = p @ vv
        mass[i] = p @ vv.abs()
        size[i] = ((kk.abs() @ q[i].abs()) * abs(scale)).max()
    return out, lse, mass, size


def attention_bounds(out, lse, mass, size, n, d, bf16):
    """What fp32 arithmetic (and bf16 weights and outputs) may differ by from the 64-bit result.  A score
    is a sum of d products, then scaled and taken in units of log2: (d + 4) roundings of at most the sum of
    its magnitudes.  A weight's relative error is that of both its score and the maximum, plus the
    exponential's; sums of n terms add n roundings."""
    delta = (d + 4) * U * size
    rel = (2 * delta + (n + 16) * U)[:, None]
    tol = rel * mass + 1e-30
    if bf16:
        tol = tol + 1.01 * U16 * mass + 1.01 * U16 * out.abs()
    return tol, delta + (n + 16) * U + 4 * U * lse.abs().nan_to_num(posinf=0.0)


def quantise(x):
    """(..., d) float64 -> the values that the 4-bit format has for them, and the scale bytes."""
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    ok = torch.isfinite(g).all(-1, keepdim=True)
    g = torch.where(ok, g, torch.zeros_like(g))
    amax = g.abs().amax(-1, keepdim=True)
    byte = torch.full_like(amax, 252.0)
    for b in range(252, 0, -1):  # the smallest byte with amax / scale < 7
        byte = torch.where(amax < 7.0 * 2.0 ** (b - 127), torch.full_like(byte, float(b)), byte)
    scale = torch.exp2(byte - 127.0)
    a = g.abs() / scale
    best = torch.zeros_like(a)
    dist = a.clone()
    for c in range(1, 8):
        dc = (a - GRID[c]).abs()
        take = (dc < dist) | ((dc == dist) & (c % 2 == 0))
        best = torch.where(take, torch.full_like(a, GRID[c]), best)
        dist = torch.minimum(dist, dc)
    return (torch.sign(g) * best * scale).reshape(x.shape), byte.squeeze(-1)
